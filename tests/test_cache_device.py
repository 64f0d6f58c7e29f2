"""Calls on a cache while another device than its own is the current one: every kernel is launched on the cache's, and the current one is as it was
afterwards.  The runtime's calls are stood in for by a small C library in a process of its own: no GPU is needed."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STAND_IN = r"""
#include <stdlib.h>
#include <string.h>
int stand_in_device = 0, stand_in_refuse = -1, stand_in_launches[4] = {0, 0, 0, 0};
int hipGetDevice(int *d) { *d = stand_in_device; return 0; }
int hipSetDevice(int d) { if (d == stand_in_refuse) return 101; stand_in_device = d; return 0; }
/* type, device: all memory is device 1's */
int hipPointerGetAttributes(int *at, const void *p) { at[0] = 2; at[1] = 1; return 0; }
int hipFuncSetAttribute(const void *f, int what, int value) { return 0; }
int __hipPushCallConfiguration(void) { return 0; }
int __hipPopCallConfiguration(void) { return 0; }
int hipLaunchKernel(const void *f, ...) { ++stand_in_launches[stand_in_device]; return 0; }
int hipGetLastError(void) { return 0; }
int hipDeviceSynchronize(void) { return 0; }
int hipHostMalloc(void **p, size_t n, unsigned flags) { *p = calloc(1, n); return 0; }
int hipHostFree(void *p) { free(p); return 0; }
int hipHostGetDevicePointer(void **d, void *h, unsigned flags) { *d = h; return 0; }
int hipEventCreateWithFlags(void **e, unsigned flags) { *e = calloc(1, 8); return 0; }
int hipEventDestroy(void *e) { free(e); return 0; }
int hipEventRecord(void *e, void *s) { return 0; }
int hipStreamWaitEvent(void *s, void *e, unsigned flags) { return 0; }
int hipStreamSynchronize(void *s) { return 0; }
int hipStreamIsCapturing(void *s, int *status) { *status = 0; return 0; }
int hipMemcpy(void *to, const void *from, size_t n, int kind) { memset(to, 0, n); return 0; }
"""

PROGRAM = r"""
import ctypes as C, sys
stand_in = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)  # in front of the runtime for every library loaded from here on
from paper_2408_02937_amd import rtams
from paper_2408_02937_amd.rtams import CacheConfig, CacheQuery, CacheSight
L = rtams.lib()
device, refuse = C.c_int.in_dll(stand_in, "stand_in_device"), C.c_int.in_dll(stand_in, "stand_in_refuse")
launches = (C.c_int * 4).in_dll(stand_in, "stand_in_launches")
cfg = CacheConfig(layers=2, kv_heads=2, head_dim=128, page_tokens=64, max_seqs=8, max_pages=4)
cfg.pool_bytes = L.rtams_cache_pool_bytes_for(C.byref(cfg), 16)
cfg.scratch_bytes = L.rtams_cache_scratch_bytes_for(C.byref(cfg))
cfg.d_pool = cfg.d_scratch = 4096  # never read: there is no device behind the runtime
at, n = 8192, C.c_int64()
query = CacheQuery(layer=0, q_heads=8, type=0, causal=1, window=0, max_new=3, scale=1.0, d_q=at, q_row_stride=1024, q_head_stride=128, d_out=at,
                   out_row_stride=1024, out_head_stride=128)
sight = CacheSight(tree_words=1, d_tree=at)
for current in (0, 1, 3):
    device.value = current
    h = C.c_void_p()
    assert L.rtams_cache_create(C.byref(cfg), C.byref(h)) == rtams.OK, L.rtams_last_error()
    calls = {
        "extend": lambda: L.rtams_cache_extend(h, 2, None, at, None), "write": lambda: L.rtams_cache_write(h, 1, 2, None, at, 6, 3, at, at, 256, 128, 0, None),
        "read": lambda: L.rtams_cache_read(h, 1, 2, None, at, 6, 3, at, at, 2, None), "attend": lambda: L.rtams_cache_attend(h, C.byref(query), 2, None, at, 6, None),
        "sight": lambda: L.rtams_cache_attend_sight(h, C.byref(query), C.byref(sight), 2, None, at, 6, None),
        "tree": lambda: L.rtams_cache_tree(h, 2, None, at, 6, 3, at, at, 1, at, None), "walk": lambda: L.rtams_cache_walk(h, 2, at, 6, 3, at, at, at, at, at, at, None),
        "keep": lambda: L.rtams_cache_keep(h, 2, None, at, 6, 3, at, at, None), "fork": lambda: L.rtams_cache_fork(h, 1, at, at, 0, None),
        "trim": lambda: L.rtams_cache_trim(h, 2, None, None, None), "compact": lambda: L.rtams_cache_compact(h, None), "clear_error": lambda: L.rtams_cache_clear_error(h)}
    for name, call in calls.items():
        before = launches[1]
        assert call() == rtams.OK, (name, L.rtams_last_error())
        assert launches[1] > before and device.value == current, (name, current, list(launches))
    assert L.rtams_cache_free_pages(h, C.byref(n)) == rtams.OK and device.value == current
    assert launches[0] == launches[2] == launches[3] == 0, (current, list(launches))
    if current == 0:  # a device that cannot be made the current one
        refuse.value = 1
        all_of = list(launches)
        for name, call in calls.items():
            if name != "clear_error":
                assert call() == rtams.EHIP and b"device 1" in L.rtams_last_error() and device.value == 0, name
        bad = C.c_void_p()
        assert L.rtams_cache_create(C.byref(cfg), C.byref(bad)) == rtams.EHIP and not bad.value
        assert list(launches) == all_of
        refuse.value = -1
    assert L.rtams_cache_destroy(h) == rtams.OK and device.value == current
print("ok")
"""


def test_kernels_are_launched_where_the_cache_is(tmp_path):
    src, lib, prog = tmp_path / "stand_in.c", tmp_path / "libstand_in.so", tmp_path / "program.py"
    src.write_text(STAND_IN)
    prog.write_text(PROGRAM)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(lib), str(src)], check=True)
    env = {**os.environ, "PYTHONPATH": ROOT, "HIP_VISIBLE_DEVICES": "-1"}
    r = subprocess.run([sys.executable, str(prog), str(lib)], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stdout + r.stderr
