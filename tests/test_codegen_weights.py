"""What the compiler makes of the loops over 4-bit weights (CPU only: hipcc writes gfx950 assembly without a GPU): their loads stay in flight."""
import functools
import os
import re
import shutil
import subprocess
import tempfile

import pytest

from paper_1511_04561_amd import build

pytestmark = pytest.mark.skipif(not (os.path.exists(build.hipcc()) or shutil.which(build.hipcc())), reason="needs hipcc")

KERNELS = """
template __global__ void k_weights_product_few<__bf16, 128, 1, 4, 4>(ProductArgs);
template __global__ void k_weights_product_few<__bf16, 32, 1, 8, 2>(ProductArgs);
template __global__ void k_weights_product<__bf16, 32, 1, 4, 1, 4, 2, 4, 5>(ProductArgs, SplitArgs);
template __global__ void k_weights_product<__bf16, 32, 4, 4, 2, 8, 1, 2, 1>(ProductArgs, SplitArgs);
template __global__ void k_weights_product<__bf16, 32, 1, 4, 1, 13, 1, 2, 4, 7>(ProductArgs, SplitArgs);
"""


@functools.lru_cache(maxsize=None)
def kernels():
    """Kernel name -> its basic blocks, lists of instructions; and -> spilled registers."""
    with tempfile.TemporaryDirectory() as d:
        src, out = os.path.join(d, "k.hip"), os.path.join(d, "k.s")
        with open(src, "w") as f:
            f.write('#include "dq8_kernels_weights.hpp"\nnamespace {\n%s}\n' % KERNELS)
        flags = [f for f in build.FLAGS if f != "-shared"]
        subprocess.check_call([build.hipcc()] + flags + ["-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "-S", "--cuda-device-only", "-o", out, src])
        text = open(out).read()
    blocks, name = {}, None
    for line in text.split("\n"):
        m = re.match(r"^_ZN12_GLOBAL__N_1\d\d(k_weights\w+):", line)
        if m:
            name = m.group(1)
            blocks[name] = [[]]
        elif line.startswith(".Lfunc_end"):
            name = None
        elif name and re.match(r"^\.LBB\w+:", line):
            blocks[name].append([])
        elif name and re.match(r"^\s+[a-z]", line):
            blocks[name][-1].append(line.split(";")[0].strip())
            if blocks[name][-1][-1].startswith("s_cbranch"):
                blocks[name].append([])
    spills = dict(re.findall(r"\.name:\s+_ZN12_GLOBAL__N_1\d\d(k_weights\w+)\n(?:.*\n)*?\s+\.vgpr_spill_count: (\d+)", text))
    return blocks, {k: int(v) for k, v in spills.items()}


def named(start, what=0):
    found = [v for k, v in kernels()[what].items() if k.startswith(start)]
    assert len(found) == 1, start
    return found[0]


def loads_left(blocks):
    """Of every block with products: how many loads its first wait for one leaves on their way."""
    got = []
    for b in blocks:
        if sum(i.startswith("v_mfma") for i in b) >= 4:
            waits = [int(m.group(1)) for i in b for m in re.finditer(r"vmcnt\((\d+)\)", i)]
            got += waits[:1]
    return got


def test_one_conversion_makes_two_operands():
    # 32 codes of a lane in a tile: 16 conversions, four products
    for start in ("k_weights_product_fewIDF16bLi128ELi1ELi4ELi4E", "k_weights_product_fewIDF16bLi32ELi1ELi8ELi2E"):
        for b in named(start):
            products = sum(i.startswith("v_mfma_f32_16x16x32_bf16") for i in b)
            assert sum(i.startswith("v_cvt_scalef32_pk_bf16_fp4") for i in b) == 4 * products


@pytest.mark.parametrize("start,tiles", [("k_weights_product_fewIDF16bLi128ELi1ELi4ELi4E", 3), ("k_weights_product_fewIDF16bLi32ELi1ELi8ELi2E", 1)])
def test_tiles_ahead_stay_on_their_way(start, tiles):
    """Codes and scales of so many tiles are not waited for when one is worked on."""
    left = loads_left(named(start))
    assert left and min(left) >= 2 * tiles, left


@pytest.mark.parametrize("start,least", [("k_weights_productIDF16bLi32ELi1ELi4ELi1ELi4ELi2ELi4ELi5E", 6), ("k_weights_productIDF16bLi32ELi4ELi4ELi2ELi8ELi1ELi2ELi1E", 4),
                                         ("k_weights_productIDF16bLi32ELi1ELi4ELi1ELi13ELi1ELi2ELi4E", 3)])
def test_chunks_ahead_stay_on_their_way(start, least):
    """Where a chunk of activations goes to LDS, behind a barrier in the loop, later chunks' loads are on their way."""
    left, code = [], [i for b in named(start) for i in b]
    barriers = [i for i, x in enumerate(code) if x == "s_barrier"] + [len(code)]
    for first, end in zip(barriers, barriers[1:]):
        part = code[first:end]
        if any(y.startswith("v_mfma") for y in part) and any(y.startswith("ds_write_b128") for y in part) and any(y.startswith("global_load") for y in part):
            left += [int(m.group(1)) for y in part for m in re.finditer(r"vmcnt\((\d+)\)", y)][:1]
    assert len(left) >= 2 and min(left) >= least, left


def test_no_spills():
    for k, v in kernels()[1].items():
        assert v == 0, k
