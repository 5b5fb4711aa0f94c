"""The paged 4-bit cache where it can go wrong besides what test_paged_fp4.py looks at: waits, threads, streams, far tails of a softmax, unusual queries,
starts and lengths."""
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2503_23294_amd as ck
from oracle import fp4_oracle as O
from paper_2503_23294_amd import _lib
from test_device_code import _objdump
from test_paged_fp4 import DTYPES, Batch, _f64

gpu = pytest.mark.gpu


# ---- shared memory of the tile kernel ----------------------------------------------------------------------------------------


def test_first_products_of_a_tile_are_done_before_their_keys_are_replaced(tmp_path):
    """The logits of a workgroup's first 32 keys are products outside the loop, and the loop's first step puts other keys in their place: between
    the two the waves have to wait for each other."""
    tool = _objdump()
    lib = shutil.copy(_lib.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([tool, "--offloading", str(lib)], cwd=tmp_path, check=True, capture_output=True)
    kernels = 0
    for obj in sorted(tmp_path.glob("lib.so.*gfx950")):
        text = subprocess.run([tool, "-d", "--no-show-raw-insn", str(obj)], check=True, capture_output=True, text=True).stdout
        for name, body in re.findall(r"^[0-9a-f]+ <(\w*fp4_tile_kernel\w*)>:\n(.*?)(?=^[0-9a-f]+ <\w+>:|\Z)", text, re.S | re.M):
            code = [line.split("//")[0].strip() for line in body.splitlines() if line.strip()]
            if not any(line.startswith("v_mfma") for line in code):
                continue
            kernels += 1
            steps = 8 if "ILi128E" in name else 4
            products = [i for i, line in enumerate(code) if line.startswith("v_mfma")][:steps]
            sums = {code[i].split()[1] for i in products}
            assert len(sums) == 1, f"{name}: the first {steps} products are not one chain: {sums}"
            behind = next(line for line in code[products[-1]:] if line.startswith(("s_barrier", "ds_write")))
            assert behind.startswith("s_barrier"), f"{name}: {behind} without a wait behind the first products"
    assert kernels == 4


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,new,kv_heads,rep", [([1100, 700], [514, 300], 4, 32),     # eight waves; 64 and 128 rows in the last tiles
                                                   ([300, 200, 90], [28, 33, 27], 2, 5),  # four waves; 12, 37 and 7 rows
                                                   ([700, 333], [683, 86], 4, 24)])       # four waves, keys not cut; 8 and 16 rows
def test_last_tiles_with_idle_waves(lens, new, kv_heads, rep, d):
    """Tiles of which at most half of the waves have rows; the same bits every time."""
    B = Batch(lens, kv_heads, d, 48, torch.float16, seed=d + rep, spread=2.0)
    B.store_all()
    q = B.query(new, rep)
    call = lambda: ck.cocktail_fp4_attention(B.cache, q, B.starts(new), max_new=max(new), max_len=max(lens))  # noqa: E731
    out, lse = call()
    B.check(q, new, out, lse)
    for _ in range(10):
        again, lse2 = call()
        assert torch.equal(out, again) and torch.equal(lse, lse2)
