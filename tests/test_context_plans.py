"""Launch rules of the observation context's operators, on the host: the plan functions are C++
symbols of the library; calling them needs no GPU."""
import ctypes

import pytest

import context_util as cu
from paper_2608_27384_amd import flashvla as fvb


def rope_tokens(n, row):
    f = getattr(fvb.lib(), "_ZN2fv11rope_tokensEim")
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_int, ctypes.c_size_t]
    return f(n, row)


# bytes of a token that are rotated or stored: a head of 64 in bf16 to three times 1024 of 256 in fp32
ROWS = [128 << i for i in range(15)] + [(6 << 10) - 16, 6 << 10, (10 << 10) - 16, 10 << 10, 12 << 10, 3 << 20]
COUNTS = [1, 2047, 2048, 16384] + [n + d for n in (1 << 23, 1 << 24, 1 << 25, 1 << 26) for d in (-1, 0, 1)]


@pytest.mark.parametrize("n", [n for n in COUNTS if n <= 1 << 26])
def test_rotary_grids_are_launches(n):
    """Every count of tokens that is taken has a grid of less than 2^32 threads of 256 a workgroup,
    which shares its angles among no more than 8 tokens."""
    for row in ROWS:
        t = rope_tokens(n, row)
        assert 1 <= t <= 8
        assert -(-n // t) * 256 < 1 << 32, (row, t)


# (tokens, bytes of one, tokens a workgroup of the fastest)
@pytest.mark.parametrize("n,row,tokens", [
    (64, 5120, 1), (4096, 5120, 2), (32768, 5120, 8), (32768, 1536, 8), (8192, 12288, 2),
    (32768, 12288, 1)])
def test_rotary_tokens_that_were_faster(n, row, tokens):
    assert rope_tokens(n, row) == tokens


# Both sides of every threshold: (type, 32-row tiles of 8 heads, mean keys, head dim, causal, kernel)
@pytest.mark.parametrize("dtype,tiles,keys,D,causal,form", [
    ("bf16", 383, 560, 256, True, cu.FEW), ("bf16", 384, 560, 256, True, cu.HALVES),
    ("bf16", 383, 9000, 64, False, cu.FEW), ("bf16", 384, 9000, 64, False, cu.HALVES),
    ("bf16", 1024, 2047, 128, True, cu.HALVES), ("bf16", 1025, 2047, 128, True, cu.TILES),
    ("bf16", 1025, 2048, 128, True, cu.HALVES), ("bf16", 2560, 2048, 192, True, cu.HALVES),
    ("bf16", 2561, 2048, 192, True, cu.TILES), ("bf16", 1024, 2048, 128, False, cu.HALVES),
    ("bf16", 1025, 2048, 128, False, cu.TILES), ("fp32", 4096, 500, 64, True, cu.FEW),
    ("fp32", 4097, 500, 64, True, cu.TILES), ("fp32", 4096, 2048, 64, True, cu.FEW),
    ("fp32", 4097, 2048, 64, True, cu.TILES), ("fp32", 4096, 2047, 192, True, cu.FEW),
    ("fp32", 4097, 2047, 256, True, cu.TILES), ("fp32", 8192, 2048, 192, False, cu.FEW),
    ("fp32", 8193, 2048, 256, True, cu.TILES), ("fp32", 2048, 2047, 128, True, cu.FEW),
    ("fp32", 2049, 2047, 128, True, cu.TILES), ("fp32", 768, 2047, 128, False, cu.FEW),
    ("fp32", 769, 2047, 128, False, cu.TILES), ("fp32", 4096, 2048, 128, False, cu.FEW),
    ("fp32", 4097, 2048, 128, True, cu.TILES)])
def test_prompt_kernels(dtype, tiles, keys, D, causal, form):
    assert cu.prompt_form(dtype, 4 * tiles, 3 * keys, 3, 8, 1, D, causal) == form


def test_direct_loads_take_their_address_register_as_an_operand():
    """The compiler keeps values in m0 of its own: a block that loads to LDS is handed m0 and
    does not set it unseen."""
    import os
    import re
    csrc = os.path.join(os.path.dirname(os.path.abspath(fvb.__file__)), "csrc")
    blocks = []
    for name in sorted(os.listdir(csrc)):
        with open(os.path.join(csrc, name)) as f:
            blocks += re.findall(r"asm volatile\(.*?\);", f.read(), re.S)
    loads = [b for b in blocks if "m0" in b or "offen lds" in b]
    assert loads and all('"{m0}"' in b and "_b32 m0" not in b for b in loads)


def test_the_gpu_tests_reach_every_prompt_kernel():
    """The shapes of the GPU tests run the kernels that they are there for, by today's choice."""
    import test_gpu_prompt_attention as t
    few = {(s[0], s[3], t.takes(s, t.LENS["ragged"], True)) for s in t.SHAPES}
    assert {f for _, _, f in few} == {cu.FEW} and {d for _, d, _ in few} == {64, 128, 192, 256}
    full = {(s[0], s[3], t.takes(s, t.LENS["ragged"], c)) for s in t.FULL for c in (True, False)}
    assert full == {(d, D, f) for d, fs in (("bf16", (cu.HALVES, cu.TILES)), ("fp32", (cu.TILES,)))
                    for D in (64, 128, 192, 256) for f in fs}
    far = {(c[0], c[3], c[5]) for c in t.FAR_CASES}
    assert far == {(d, D, f) for d, fs in (("bf16", (cu.FEW, cu.HALVES, cu.TILES)), ("fp32", (cu.FEW, cu.TILES)))
                   for D in (64, 128, 192, 256) for f in fs}
