"""Attention over a cache in 8 bits against the 64-bit form of what its codes stand for: one token a
sequence and several, lengths from zero to many chunks, page sizes that end inside a tile, groups of
one to more than sixteen heads, places that hold no keys, offsets that do not ascend, what a query
does not see."""
import numpy as np
import pytest

import context_util as cu
import quant_util as qu
from test_quant_refusals import part_plan

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", 8, 1, 256), ("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("bf16", 6, 2, 192),
          ("bf16", 40, 2, 128), ("fp32", 4, 2, 64), ("fp32", 2, 1, 256), ("fp32", 3, 3, 192),
          ("fp32", 34, 2, 128)]
IDS = dict(ids=lambda s: "x".join(map(str, s)))
LENS = [0, 1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 700, 2049]


def check(shape, cache, table, lens, q, out, layer, seqs=None):
    for i, b in enumerate(range(len(lens)) if seqs is None else seqs):
        k, v = qu.context(cache, table, b, lens[b], layer)
        cu.check_attention_wide(out[i:i + 1], qu.attention(q[i:i + 1], k, v, [lens[b]], shape[0]), shape[0])


def codes_at(cache, pool, values, layer, page, row, fn):
    """Changes the codes (uint8 [G, D]) of one position through fn."""
    x = qu.rows_of(pool[layer], values)
    x[page, :, row] = fn(x[page, :, row])
    pool[layer].copy_(qu.stored(x, values))


# ------------------------------------------------------------------ one token a sequence

@pytest.mark.parametrize("page_len", [16, 48, 128])
@pytest.mark.parametrize("max_len", [0, 2049, 40])
@pytest.mark.parametrize("shape", SHAPES, **IDS)
def test_tokens_against_the_definition(shape, page_len, max_len):
    torch = cu.torch_mod()
    cache, q, table = qu.make(shape, LENS, page_len, extra=7)
    out = torch.full_like(q, 7.0)
    cache.attend(1, q, cu.ints(np.arange(len(LENS))), out, max_len=max_len)
    check(shape, cache, table, LENS, q, out, 1)
    assert not out[0].any()


@pytest.mark.parametrize("page_len", [16, 240, 256])
@pytest.mark.parametrize("shape", [SHAPES[2], SHAPES[5]], **IDS)
def test_every_page_length(shape, page_len):
    torch = cu.torch_mod()
    lens = [0, 1, page_len - 1, page_len, page_len + 1, 3 * page_len + 17, 4000 + page_len]
    cache, q, table = qu.make(shape, lens, page_len, extra=2)
    for max_len in (0, 100):
        out = torch.full_like(q, 7.0)
        cache.attend(1, q, cu.ints(range(len(lens))), out, max_len=max_len)
        check(shape, cache, table, lens, q, out, 1)


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[4], SHAPES[5]], **IDS)
def test_one_row_long_context(shape):
    torch = cu.torch_mod()
    cache, q, table = qu.make(shape, [20011], 16, layers=1)
    out = torch.full_like(q, 7.0)
    cache.attend(0, q, cu.ints([0]), out)
    check(shape, cache, table, [20011], q, out, 0)


@pytest.mark.parametrize("spread", [20, 100])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[5]], **IDS)
def test_scales_far_apart(shape, spread):
    """Blocks whose scales differ by up to 2^40 and 2^200 in the values, near one in the keys."""
    torch = cu.torch_mod()
    lens = [300, 77]
    cache, q, table = qu.make(shape, lens, layers=1, spread=spread)
    cache.k_scale.view(torch.uint8).copy_(cache.k_scale.view(torch.uint8).clamp(118, 122))
    for part in (False, True):
        out = torch.full_like(q, 7.0)
        if part:
            cache.attend_part(0, q, cu.ints([0, 1, 2]), cu.ints([0, 1]), out)
        else:
            cache.attend(0, q, cu.ints([0, 1]), out)
        for b, n in enumerate(lens):
            k, v = qu.context(cache, table, b, n, 0)
            ref = qu.attention(q[b:b + 1], k, v, [n], shape[0])
            (cu.check_attention if part else cu.check_attention_wide)(out[b:b + 1], ref, shape[0])


@pytest.mark.parametrize("shape", [SHAPES[1], SHAPES[6]], **IDS)
def test_padded_rows_repeats_and_strides(shape):
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    lens = [300, 5, 70]
    cache, _, table = qu.make(shape, lens)
    seqs = [2, -1, 0, 0, 3, 1, 65536]
    wide = cu.randn(dtype, 9, len(seqs), H * D + 64)
    q = wide[:, :H * D].unflatten(1, (H, D))
    for part in (False, True):
        full = torch.full((len(seqs), H * D + 32), 7.0, dtype=q.dtype, device="cuda")
        out = full[:, :H * D].unflatten(1, (H, D))
        if part:
            cache.attend_part(0, q, cu.ints(range(8)), cu.ints(seqs), out, causal=False)
        else:
            cache.attend(0, q, cu.ints(seqs), out)
        for i, b in enumerate(seqs):
            if 0 <= b < 3:
                k, v = qu.context(cache, table, b, lens[b], 0)
                cu.check_attention(out[i:i + 1], qu.attention(q[i:i + 1], k, v, [lens[b]], dtype), dtype)
            else:
                assert (out[i] == 7).all()
        assert (full[:, H * D:] == 7).all()


@pytest.mark.parametrize("max_len", [0, 30])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[2], SHAPES[7]], **IDS)
def test_entries_that_are_no_page_hold_no_keys(shape, max_len):
    torch = cu.torch_mod()
    lens = [200, 100, 64, 40]
    cache, q, table = qu.make(shape, lens)
    holes = {0: [3, 7], 1: [0], 2: [0, 1, 2, 3], 3: [1, 2]}
    for b, cols in holes.items():
        for j, c in enumerate(cols):
            cache.table[b, c] = (-1, 1 << 20, -(1 << 31), cache.c.n_pages)[j % 4]
    for part in (False, True):
        out = torch.full_like(q, 7.0)

        def call():
            if part:
                cache.attend_part(0, q, cu.ints(range(5)), cu.ints(range(4)), out, max_len=max_len)
            else:
                cache.attend(0, q, cu.ints(range(4)), out, max_len=max_len)

        call()
        for b, cols in holes.items():
            k, v = qu.context(cache, table, b, lens[b], 0)
            keep = [i for i in range(lens[b]) if i // 16 not in cols]
            cu.check_attention(out[b:b + 1], qu.attention(q[b:b + 1], k[keep], v[keep], [len(keep)], shape[0]), shape[0])
        assert not out[2].any()
        cache.length.fill_(1 << 30)  # longer than the table: what the table holds
        cache.length[0] = -5
        call()
        assert not out[0].any()
        cache.length.copy_(cu.ints(lens))


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[5]], **IDS)
def test_keys_and_queries_that_are_not_finite(shape):
    """A NaN key of one that is seen, infinite queries: NaN, in the heads that read it."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    lens = [400, 400, 400]
    cache, q, table = qu.make(shape, lens, layers=1)
    codes_at(cache, cache.k, False, 0, table[0, 17 // 16], 17 % 16, lambda x: x.fill_(127))
    q[1, 0, 5] = np.inf
    for part in (False, True):
        out = torch.full_like(q, 7.0)
        if part:
            cache.attend_part(0, q, cu.ints(range(4)), cu.ints(range(3)), out)
        else:
            cache.attend(0, q, cu.ints(range(3)), out)
        assert out[0].isnan().all() and out[1, 0].isnan().all()
        k, v = qu.context(cache, table, 2, 400, 0)
        cu.check_attention(out[2:], qu.attention(q[2:], k, v, [400], dtype), dtype)
        k, v = qu.context(cache, table, 1, 400, 0)
        cu.check_attention(out[1:2, 1:], tuple(x[:, 1:] for x in qu.attention(q[1:2].nan_to_num(0, 0, 0), k, v, [400], dtype)), dtype)


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[2], SHAPES[5]], **IDS)
def test_values_that_are_not_numbers(shape):
    torch = cu.torch_mod()
    lens = [1, 40, 700, 2049]
    cache, q, table = qu.make(shape, lens, layers=1)
    for b, n in enumerate(lens):
        for at, d in ((0, 3), (n - 1, 5), (n // 2, 7)):
            def put(x, d=d):
                x[:, d] = 255
                return x
            codes_at(cache, cache.v, True, 0, table[b, at // 16], at % 16, put)
    hit = torch.zeros(shape[3], dtype=torch.bool, device="cuda")
    hit[[3, 5, 7]] = True
    for part in (False, True):
        out = torch.full_like(q, 7.0)
        if part:
            cache.attend_part(0, q, cu.ints(range(5)), cu.ints(range(4)), out)
        else:
            cache.attend(0, q, cu.ints(range(4)), out)
        assert out[..., hit].isnan().all() and out[..., ~hit].isfinite().all()


def test_two_graphs_and_growing_lengths():
    """Captured calls replayed on two streams at once keep workspaces of their own, and follow the
    lengths that the cache holds when they run."""
    torch = cu.torch_mod()
    shape = SHAPES[1]
    lens = [1500, 900]
    cache, q, table = qu.make(shape, lens)
    seqs, cum = cu.ints([0, 1]), cu.ints([0, 1, 2])
    calls = [lambda out: cache.attend(0, q, seqs, out, max_len=1500),
             lambda out: cache.attend_part(1, q, cum, seqs, out, max_len=1500)]
    outs, graphs = [], []
    for call in calls:
        out = torch.zeros_like(q)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(out)
        outs.append(out)
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for now in ([1500, 900], [17, 0], [1499, 128]):
        cache.length.copy_(cu.ints(now))
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for layer, call in enumerate(calls):
            for b, n in enumerate(now):
                k, v = qu.context(cache, table, b, n, layer)
                cu.check_attention(outs[layer][b:b + 1], qu.attention(q[b:b + 1], k, v, [n], "bf16"), "bf16")
            eager = torch.zeros_like(q)
            call(eager)
            assert torch.equal(eager, outs[layer])


def test_a_row_does_not_depend_on_the_others():
    torch = cu.torch_mod()
    shape = SHAPES[0]
    cache, q, table = qu.make(shape, [800, 40, 333])
    a, b = torch.zeros_like(q), torch.zeros_like(q)
    cache.attend(0, q, cu.ints([0, 1, 2]), a)
    cache.length[0] = 3
    cache.attend(0, q, cu.ints([0, 1, 2]), b)
    assert torch.equal(a[1:], b[1:]) and not torch.equal(a[0], b[0])


@pytest.mark.parametrize("shape", [(t, 4, 4, D) for t in ("bf16", "fp32") for D in (64, 128, 192, 256)], **IDS)
def test_more_than_the_caches_hold(shape):
    """A layer of more than half a gigabyte, and rows that might read as much: streamed."""
    torch = cu.torch_mod()
    from paper_2608_27384_amd.flashvla import QuantCache
    small, q, table = qu.make(shape, LENS, layers=1)
    pages = (1 << 29) // (16 * 2 * shape[2] * shape[3]) + 7
    columns = min(pages, 65536)
    cache = QuantCache.empty(1, shape[2], shape[3], pages, len(LENS), columns, 16, cu.ttype(shape[0]))
    for a, b in zip(cache.pools, small.pools):
        a, b = a.view(torch.uint8), b.view(torch.uint8)
        a.fill_(255)
        a[:, :b.shape[1]] = b
    wide = np.full((len(LENS), columns), -1)
    wide[:, :table.shape[1]] = table
    cache.table.copy_(cu.ints(wide))
    cache.length.copy_(cu.ints(LENS))
    for max_len in (0, pages * 16):
        out = torch.full_like(q, 7.0)
        cache.attend(0, q, cu.ints(range(len(LENS))), out, max_len=max_len)
        check(shape, cache, table, LENS, q, out, 0)


def one_hot(shape, lens, page_len, layers=1):
    """Queries of zero, and the value of position p in kv head g a one at element (p + g) % D."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    cache, q, table = qu.make(shape, lens, page_len, layers=layers)
    rows = qu.rows_of(cache.v, True)
    rows[(rows & 127) != 127] = 0
    g = torch.arange(G, device="cuda")[:, None]
    for b, n in enumerate(lens):
        for j in range(-(-n // page_len)):
            p = torch.arange(page_len * j, min(page_len * j + page_len, n), device="cuda")[None]
            for l in range(layers):
                rows[l, table[b, j], :, :p.shape[1]] = rows[l, table[b, j], :, :p.shape[1]].scatter(
                    2, ((p + g) % D)[..., None], 56)  # the code of 1
    cache.v.copy_(qu.stored(rows, True))
    s = cache.v_scale.view(torch.uint8)
    s[s != 255] = 127
    return cache, q.zero_(), table


def counts(n, D, H, G):
    """How many of n positions fall on each element, [..., H, D]."""
    torch = cu.torch_mod()
    d, h = torch.arange(D, device="cuda"), (torch.arange(H, device="cuda") * G // H)[:, None]
    return torch.div(n[..., None, None] - (d - h) % D + D - 1, D, rounding_mode="floor").clamp(min=0)


@pytest.mark.parametrize("max_len", [0, 4900, 40])
@pytest.mark.parametrize("shape", SHAPES, **IDS)
def test_every_key_counts_once(shape, max_len):
    """Every probability is one: a row's result is, times its length, how many positions fall on
    each element.  Sums of ones stay within 2^-16 (each of at most 77 additions, and of a lane's 20
    by 64 lanes and 39 chunks for the denominator, off by 2^-24); with the result's own rounding
    that leaves less than half a key."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    lens = [1, 16, 127, 128, 129, 1000, 2048, 3333, 4900]
    cache, q, table = one_hot(shape, lens, 48)
    n = torch.tensor(lens, device="cuda")
    want = counts(n, D, H, G)
    for part in (False, True):
        out = torch.full_like(q, 7.0)
        if part:
            cache.attend_part(0, q, cu.ints(range(10)), cu.ints(range(9)), out, max_len=max_len)
        else:
            cache.attend(0, q, cu.ints(range(9)), out, max_len=max_len)
        assert bool(((out.double() * n[:, None, None] - want).abs() <= want * (cu.EPS[dtype] + 2.0 ** -16)).all())


@pytest.mark.parametrize("shape,n,keys", [(("bf16", 8, 1, 256), 1, 448), (("fp32", 2, 1, 256), 1, 256),
                                          (("bf16", 8, 1, 256), 64, 768), (("bf16", 4, 4, 64), 32, 2048),
                                          (("fp32", 4, 4, 64), 32, 2048)])
def test_one_chunk_and_several(shape, n, keys):
    """The longest sequences that one workgroup walks, and the next longer ones."""
    torch = cu.torch_mod()
    for top in (keys, keys + 1):
        lens = [top - 37 * b % top for b in range(n)]
        cache, q, table = qu.make(shape, lens, layers=1)
        out = torch.full_like(q, 7.0)
        cache.attend(0, q, cu.ints(range(n)), out, max_len=top)
        check(shape, cache, table, lens, q, out, 0)


# ------------------------------------------------------------------ several tokens a sequence

def entries(parts, cut=()):
    """cu_q of entries of these many rows."""
    return np.cumsum([0] + list(parts))


def check_parts(shape, cache, table, lens, seqs, cum, q, out, layer, causal):
    for i, b in enumerate(seqs):
        lo, hi = cum[i], cum[i + 1]
        if not 0 <= b < len(lens):
            assert (out[lo:hi] == 7).all()
            continue
        k, v = qu.context(cache, table, b, lens[b], layer)
        m = hi - lo
        limits = [max(0, lens[b] - m + j + 1) if causal else lens[b] for j in range(m)]
        cu.check_attention(out[lo:hi], qu.attention(q[lo:hi], k, v, limits, shape[0]), shape[0])
    assert (out[cum[-1]:] == 7).all()


PARTS = [  # (lengths, rows of each entry, sequence of each entry)
    ([40, 300, 17, 0, 1, 129, 33], [3, 50, 17, 4, 1, 129, 40], [0, 1, 2, 3, 4, 5, 6]),
    ([1000, 16, 250], [1, 0, 9, 30, 2, 5], [0, 1, -1, 2, 3, 0]),
    ([2500], [77], [0])]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("page_len,max_len", [(16, 0), (48, 2500), (128, 50)])
@pytest.mark.parametrize("shape", SHAPES, **IDS)
def test_parts_against_the_definition(shape, page_len, max_len, causal):
    """More queries than keys among them (the first rows of a causal part see none: zeros), rows
    that no entry has, a sequence twice, entries without rows and without a sequence."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    for x, (lens, rows, seqs) in enumerate(PARTS):
        cache, _, table = qu.make(shape, lens, page_len, seed=x, extra=3)
        cum = entries(rows)
        q = cu.randn(dtype, 50 + x, int(cum[-1]) + 3, H, D)
        out = torch.full_like(q, 7.0)
        cache.attend_part(1, q, cu.ints(cum), cu.ints(seqs), out, causal=causal, max_len=max_len)
        check_parts(shape, cache, table, lens, seqs, cum, q, out, 1, causal)


MANY = [("bf16", 8, 1, 256), ("bf16", 32, 8, 128), ("bf16", 8, 2, 64), ("bf16", 4, 2, 192),
        ("fp32", 8, 1, 256), ("fp32", 8, 2, 128), ("fp32", 4, 2, 64), ("fp32", 4, 2, 192)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", MANY, **IDS)
def test_parts_of_many_rows(shape, causal):
    """Enough rows to fill the chip by themselves, over keys that end inside tiles and blocks."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    lens, rows, seqs = [2300, 700, 515, 90], [2100, 333, 515, 120], [0, 1, 2, 3]
    rows = [-(-r * 8 // H) if H > 8 else r for r in rows]
    cache, _, table = qu.make(shape, lens, 32, layers=1)
    cum = entries(rows)
    q = cu.randn(dtype, 4, int(cum[-1]), H, D)
    out = torch.full_like(q, 7.0)
    cache.attend_part(0, q, cu.ints(cum), cu.ints(seqs), out, causal=causal, max_len=2300)
    check_parts(shape, cache, table, lens, seqs, cum, q, out, 0, causal)


@pytest.mark.parametrize("rows", [5, 300, 1500])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1], SHAPES[2], SHAPES[3], SHAPES[5], SHAPES[6], SHAPES[7], SHAPES[8]], **IDS)
def test_every_key_that_is_seen_counts_once(shape, rows):
    """Causal rows with all probabilities one: each counts its own keys.  In bf16 an unrounded one is
    one; see test_every_key_counts_once for the sums."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    n = 1700
    cache, _, table = one_hot(shape, [n], 48)
    q = torch.zeros(rows, H, D, dtype=cu.ttype(dtype), device="cuda")
    for max_len in (0, n, 100):
        out = torch.full_like(q, 7.0)
        cache.attend_part(0, q, cu.ints([0, rows]), cu.ints([0]), out, max_len=max_len)
        see = torch.arange(n - rows + 1, n + 1, device="cuda")
        want = counts(see, D, H, G)
        assert bool(((out.double() * see[:, None, None] - want).abs() <= want * (cu.EPS[dtype] + 2.0 ** -16)).all())


def in_one_chunk(shape, rows):
    """New tokens of one sequence, and a bound of its length, that make one chunk of row tiles of `rows`."""
    dtype, H, G, D = shape
    from paper_2608_27384_amd import flashvla as fvb
    for m in (3, 500, 600, 1100, 2500, 4000, 60000 // H, 120000 // H):
        for top in (100, 9013):
            p = part_plan(m, 1, H, G, D, top, fvb.FV_BF16 if dtype == "bf16" else fvb.FV_FP32)
            if (p.rows, p.n_chunks) == (rows, 1):
                return m, top


@pytest.mark.parametrize("holes", [False, True])
@pytest.mark.parametrize("rows", [32, 64, 128])
@pytest.mark.parametrize("shape", MANY, **IDS)
def test_long_walks(shape, rows, holes):
    """More keys than a workgroup looks up blocks for at once, in one chunk, by each of the kernels.
    All probabilities are one, see test_every_key_counts_once: here up to 9013 keys by at most 141
    steps of 64 of them, a lane's 16 after another, so sums are off by 2^-24 for each of at most 2^8 +
    16 additions."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    n, page_len = 9013, 48
    m, max_len = in_one_chunk(shape, rows)
    cache, _, table = one_hot(shape, [n], page_len)
    there = torch.ones(n, dtype=torch.bool, device="cuda")
    if holes:
        for i, col in enumerate((0, 7, 87, 88, 90, 120, 187)):
            cache.table[0, col] = (-1, cache.c.n_pages)[i % 2]
            there[col * page_len:(col + 1) * page_len] = False
    q = torch.zeros(m, H, D, dtype=cu.ttype(dtype), device="cuda")
    out = torch.full_like(q, 7.0)
    cache.attend_part(0, q, cu.ints([0, m]), cu.ints([0]), out, max_len=max_len)
    limits = torch.arange(n - m + 1, n + 1, device="cuda").clamp(min=0)
    see = torch.cat([there.new_zeros(1, dtype=torch.long), there.long().cumsum(0)])[limits]
    for g in range(G):
        hot = torch.nn.functional.one_hot((torch.arange(n, device="cuda") + g) % D, D) * there[:, None]
        want = torch.cat([hot.new_zeros(1, D), hot.cumsum(0)])[limits][:, None].double()
        got = out[:, g * H // G:(g + 1) * H // G].double()
        assert bool(((got * see[:, None, None] - want).abs() <= want * (cu.EPS[dtype] + 2.0 ** -15)).all())


@pytest.mark.parametrize("rows", [32, 64, 128])
@pytest.mark.parametrize("shape", MANY, **IDS)
def test_a_part_repeats_itself(shape, rows):
    """Several workgroups on every CU, a missing page and the last keys inside a tile: the same bits
    from every call, whatever runs beside it."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    from paper_2608_27384_amd import flashvla as fvb
    t = fvb.FV_BF16 if dtype == "bf16" else fvb.FV_FP32
    plans = {top: m for top in (0, 100, 1500) for m in (40, 300, 1000, 2000, 4000, 8000, 16000, 32000)
             if part_plan(m, 1, H, G, D, top or 1504, t).rows == rows}
    cache, _, table = qu.make(shape, [1500], 16, layers=1)
    cache.table[0, 30] = -1
    assert plans
    for top, m in plans.items():
        q = cu.randn(dtype, 5, m, H, D)
        calls = []
        for _ in range(4):
            out = torch.full_like(q, 7.0)
            cache.attend_part(0, q, cu.ints([0, m]), cu.ints([0]), out, causal=False, max_len=top)
            calls.append(out)
        for out in calls:
            assert out.isfinite().all() and out.equal(calls[0])


HOLES = [(16, [5, 10, 30]), (48, [3, 4, 9])]  # page_len, table columns that are no page


def nan_values(shape, cache, table, n, page_len, cols):
    """NaN in values beside missing blocks, in the same 32 keys and behind: {position: element}."""
    gone = {p // 16 for c in cols for p in range(c * page_len, (c + 1) * page_len, 16)}
    at = {}
    for b in sorted({x ^ 1 for x in gone} | {0, n // 32 * 2 - 4}):
        if b in gone or 16 * b + 16 > n:
            continue
        p, d = 16 * b + (7 * b + 3) % 16, (11 * b + 5) % shape[3]
        at[p] = d

        def put(x, d=d):
            x[:, d] = 255
            return x
        codes_at(cache, cache.v, True, 0, table[0, p // page_len], p % page_len, put)
    return at


@pytest.mark.parametrize("page_len,cols", HOLES, ids=lambda x: str(x) if isinstance(x, int) else None)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("rows", [32, 64, 128, "chunks"])
@pytest.mark.parametrize("shape", MANY, **IDS)
def test_values_that_are_not_numbers_beside_missing_pages(shape, rows, causal, page_len, cols):
    """In each kernel: NaN in the element of a value, in the rows that see it and no others, where the
    other 16 of its 32 keys have no page; every other element keeps its bits."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    m, max_len = (40, 0) if rows == "chunks" else in_one_chunk(shape, rows)
    n = 1500
    cache, _, table = qu.make(shape, [n], page_len, layers=1)
    for c in cols:
        cache.table[0, c] = -1
    q = cu.randn(dtype, 8, m, H, D)

    def run():
        out = torch.full_like(q, 7.0)
        cache.attend_part(0, q, cu.ints([0, m]), cu.ints([0]), out, causal=causal, max_len=max_len)
        return out

    clean = run()
    assert clean.isfinite().all()
    at = nan_values(shape, cache, table, n, page_len, cols)
    assert len(at) >= 4
    got = run()
    limits = torch.arange(n - m + 1, n + 1, device="cuda").clamp(min=0) if causal else torch.full((m,), n, device="cuda")
    want = torch.zeros(m, 1, D, dtype=torch.bool, device="cuda")
    for p, d in at.items():
        want[:, 0, d] |= limits > p
    assert got.isnan().equal(want.expand(m, H, D))
    assert got[~got.isnan()].equal(clean[~got.isnan()])


@pytest.mark.parametrize("max_len", [0, 100])
@pytest.mark.parametrize("page_len,cols", HOLES, ids=lambda x: str(x) if isinstance(x, int) else None)
@pytest.mark.parametrize("shape", SHAPES, **IDS)
def test_a_token_sees_values_that_are_not_numbers_beside_missing_pages(shape, page_len, cols, max_len):
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    n = 1500
    cache, q, table = qu.make(shape, [n], page_len, layers=1)
    for c in cols:
        cache.table[0, c] = -1
    clean, got = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
    cache.attend(0, q, cu.ints([0]), clean, max_len=max_len)
    assert clean.isfinite().all()
    at = nan_values(shape, cache, table, n, page_len, cols)
    cache.attend(0, q, cu.ints([0]), got, max_len=max_len)
    want = torch.zeros(D, dtype=torch.bool, device="cuda")
    want[list(at.values())] = True
    assert got.isnan().equal(want.expand(1, H, D))
    assert got[..., ~want].equal(clean[..., ~want])


@pytest.mark.parametrize("m,n,max_len", [(1, 300, 0), (17, 866, 0), (50, 866, 866), (40, 1500, 100)])
@pytest.mark.parametrize("shape", [("bf16", 8, 1, 256), ("bf16", 8, 2, 64), ("bf16", 4, 2, 192), ("bf16", 8, 4, 128)], **IDS)
def test_few_rows_keep_16_bits_of_their_probabilities(shape, m, n, max_len):
    """The kernel of 32 rows, in chunks and in one, to what two parts of a probability leave."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    assert part_plan(m, 1, H, G, D, max_len or -(-n // 16) * 16).rows == 32
    cache, _, table = qu.make(shape, [n], layers=1)
    q = cu.randn(dtype, 12, m, H, D)
    out = torch.full_like(q, 7.0)
    cache.attend_part(0, q, cu.ints([0, m]), cu.ints([0]), out, max_len=max_len)
    k, v = qu.context(cache, table, 0, n, 0)
    cu.check_attention_wide(out, qu.attention(q, k, v, [n - m + 1 + j for j in range(m)], dtype), dtype)


@pytest.mark.parametrize("n", [62, 63, 64, 65, 300])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[5]], **IDS)
def test_many_entries(shape, n):
    """Entries of no row to 40, of which neighbours share a workgroup's slots."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    lens = [1 + 53 * b % 200 for b in range(20)]
    rows = [b * b % 41 if b % 7 else 0 for b in range(n)]
    seqs = [b * 3 % 21 - (b % 11 == 0) for b in range(n)]
    cache, _, table = qu.make(shape, lens, 16)
    cum = entries(rows)
    q = cu.randn(dtype, n, int(cum[-1]), H, D)
    out = torch.full_like(q, 7.0)
    cache.attend_part(1, q, cu.ints(cum), cu.ints(seqs), out)
    check_parts(shape, cache, table, lens, seqs, cum, q, out, 1, True)


@pytest.mark.parametrize("max_len", [0, 1300])
@pytest.mark.parametrize("rows", [7, 40, 600])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1], SHAPES[2], SHAPES[3], SHAPES[5], SHAPES[6], SHAPES[7]], **IDS)
def test_what_is_not_seen_has_no_influence(shape, rows, max_len):
    """The last positions hold NaN and numbers of other sizes: every bit of the rows that do not see
    them stays; the rows that see a NaN value have NaN in its element and no other."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    n = 1300
    cache, _, table = qu.make(shape, [n], 16, layers=1)
    q = cu.randn(dtype, 6, rows, H, D)

    def run():
        out = torch.full_like(q, 7.0)
        cache.attend_part(0, q, cu.ints([0, rows]), cu.ints([0]), out, max_len=max_len)
        return out

    clean = run()
    late = n - rows // 2  # positions that the first half of the rows does not see
    for p in (late, n - 1):
        def put(x):
            x[:, 9] = 127
            x[:, D - 2] = 0x77
            return x
        codes_at(cache, cache.v, True, 0, table[0, p // 16], p % 16, put)
        codes_at(cache, cache.k, False, 0, table[0, p // 16], p % 16, lambda x: x.random_(0, 120))
    got = run()
    first = late - (n - rows)  # the first row that sees `late`
    assert got[:first].equal(clean[:first])
    assert got[first:, :, 9].isnan().all()
    rest = torch.ones(D, dtype=torch.bool, device="cuda")
    rest[9] = False
    assert got[first:][..., rest].isfinite().all()


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[5]], **IDS)
def test_offsets_that_do_not_ascend(shape):
    """Wrong offsets stay inside the tensors: rows of no entry's and past the last are not written
    where offsets ascend behind them, and the right entries of a list with a wrong one are right."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    lens = [60, 200]
    cache, _, table = qu.make(shape, lens)
    q = cu.randn(dtype, 3, 64, H, D)
    for cum in ([0, 70, 90], [5, 3, 1], [-7, 20, 64], [0, -3, 64], [64, 64, 64], [1 << 30, 1 << 30, 1 << 30]):
        out = torch.full_like(q, 7.0)
        cache.attend_part(0, q, cu.ints(cum), cu.ints([0, 1]), out)
        torch.cuda.synchronize()
    out = torch.full_like(q, 7.0)
    cache.attend_part(0, q, cu.ints([10, 30, 50]), cu.ints([0, 1]), out)  # from row 10 on
    assert (out[:10] == 7).all() and (out[50:] == 7).all()
    for i, b in enumerate((0, 1)):
        lo = 10 + 20 * i
        k, v = qu.context(cache, table, b, lens[b], 0)
        ref = qu.attention(q[lo:lo + 20], k, v, [lens[b] - 19 + j for j in range(20)], dtype)
        cu.check_attention(out[lo:lo + 20], ref, dtype)


@pytest.mark.parametrize("rows,max_len", [(64, 0), (64, 100), (2000, 100)])
@pytest.mark.parametrize("entries", [2, 70])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[5], ("bf16", 32, 8, 128)], **IDS)
def test_wrong_offsets_write_no_other_rows(shape, entries, rows, max_len):
    """Between guard rows, which offsets outside the rows or descending leave as they were; so they do
    all rows where no entry has any."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    lens = [60, 200]
    cache, _, table = qu.make(shape, lens)
    q = cu.randn(dtype, 3, rows, H, D)
    full = torch.full((rows + 512, H, D), 7.0, dtype=q.dtype, device="cuda")
    out = full[256:256 + rows]
    big, mid = 1 << 30, rows // 3
    for first, last in ((rows, rows), (big, big), (5, 1), (rows, 0), (-9, -9), (-big, -1), (rows + 1, big),  # no rows
                        (0, rows + 6), (-7, rows), (-big, big), (mid, big)):
        for middle in (first, last, (first + last) // 2):
            cum = [first] + [middle] * (entries - 1) + [last]
            cache.attend_part(0, q, cu.ints(cum), cu.ints([i % 2 for i in range(entries)]), out, max_len=max_len)
            assert (full[:256] == 7).all() and (full[256 + rows:] == 7).all()
            begin, end = (min(max(x, 0), rows) for x in (first, last))
            assert (out[:begin] == 7).all()
            if begin >= end:
                assert (out == 7).all()
            else:
                assert (out[begin:end] != 7).any(-1).all() and out.isfinite().all()
            out.fill_(7.0)


def test_nothing_to_attend():
    torch = cu.torch_mod()
    cache, q, _ = qu.make(SHAPES[2], [10, 20])
    none = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    cache.attend_part(0, none, cu.ints([0]), cu.ints([]), none.clone())
    cache.attend_part(0, none, cu.ints([0, 0]), cu.ints([1]), none.clone())
    cache.attend(0, none, cu.ints([]), none.clone())
    out = torch.full_like(q, 7.0)
    cache.attend_part(0, q, cu.ints([0]), cu.ints([]), out)
    assert (out == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_part_of_one_token_is_a_token(dtype):
    """Both attentions of one token a sequence, to what their probabilities keep."""
    torch = cu.torch_mod()
    shape = (dtype, 8, 2, 128)
    lens = [1, 50, 900, 333]
    cache, q, table = qu.make(shape, lens)
    a, b = torch.empty_like(q), torch.empty_like(q)
    cache.attend(0, q, cu.ints(range(4)), a)
    cache.attend_part(0, q, cu.ints(range(5)), cu.ints(range(4)), b)
    for i, n in enumerate(lens):
        k, v = qu.context(cache, table, i, n, 0)
        ref = qu.attention(q[i:i + 1], k, v, [n], dtype)
        cu.check_attention_wide(a[i:i + 1], ref, dtype)
        cu.check_attention(b[i:i + 1], ref, dtype)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c = torch.empty_like(q)
    seqs, cum = cu.ints(range(4)), cu.ints(range(5))
    torch.cuda.synchronize()
    cache.attend_part(0, q, cum, seqs, c, stream=s)
    s.synchronize()
    assert c.equal(b)
