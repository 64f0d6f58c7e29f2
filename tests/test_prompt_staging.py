"""How the codes of the cache come to LDS in the attention of many rows, read from the built library: by copies where that is faster, by loads
into registers elsewhere.  No GPU is needed."""
import re
import subprocess

from paper_2408_02937_amd import build
from tests.test_kernel_resources import code_objects


def test_codes_come_by_copies_where_that_is_faster(tmp_path):
    """Copies take 3 % from prompts without a sight at 64 channels, and cost up to 4 % at 128 and 2.5 % at 256."""
    with open(build.LIB, "rb") as f:
        images = [e for e in code_objects(f.read()) if b"k_cache_promptI" in e]
    assert len(images) == 1
    image = tmp_path / "prompt.elf"
    image.write_bytes(images[0])
    text = subprocess.run(["/opt/rocm/llvm/bin/llvm-objdump", "-d", "--no-show-raw-insn", str(image)], capture_output=True, text=True, check=True).stdout
    parts = re.split(r"^[0-9a-f]+ <(\w+)>:$", text, flags=re.M)
    copies = {name: "global_load_lds_dwordx4" in code for name, code in zip(parts[1::2], parts[2::2]) if "k_cache_prompt" in name}
    assert len(copies) == 11
    assert {int(re.search(r"k_cache_promptILi(\d+)E", n)[1]): c for n, c in copies.items() if "k_cache_promptI" in n} == {64: True, 96: False, 128: False, 256: False}
    assert all(c for n, c in copies.items() if "k_cache_prompt_sight" in n)
