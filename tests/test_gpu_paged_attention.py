"""Attention over the paged cache against the 64-bit form: lengths from zero to
many chunks, page sizes that end inside a tile, groups of one to more than
sixteen heads, places that hold no keys, offsets past 32 bits."""
import numpy as np
import pytest

import context_util as cu

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", 8, 1, 256), ("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("bf16", 6, 2, 192),
          ("bf16", 40, 2, 128), ("fp32", 4, 2, 64), ("fp32", 2, 1, 256), ("fp32", 3, 3, 192),
          ("fp32", 34, 2, 128)]
LENS = [0, 1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 700, 2049]


def make(shape, lens, page_len=16, seed=0, layers=2, extra=0):
    """A cache with scattered pages; everything that holds no token is NaN."""
    from paper_2608_27384_amd.flashvla import PageCache
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    need = [-(-n // page_len) for n in lens]
    total, width = sum(need) + 5, max(max(need), 1) + extra
    ids = np.random.default_rng(seed).permutation(total)
    table = np.full((len(lens), width), -1)
    at, refs = 0, np.zeros(total)
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    refs[ids[:at]] = 1
    k, v = (cu.randn(dtype, seed + i, layers, total, G, page_len, D) for i in (1, 2))
    live = torch.zeros(total, page_len, dtype=torch.bool)
    for b, n in enumerate(lens):
        for j in range(need[b]):
            live[table[b, j], :min(page_len, n - j * page_len)] = True
    for x in (k, v):
        x.masked_fill_(~live.cuda()[None, :, None, :, None], float("nan"))
    cache = PageCache(k, v, cu.ints(table), cu.ints(lens), cu.ints(refs))
    return cache, cu.randn(dtype, seed + 3, len(lens), H, D), table


def rows(cache, table, b, n, layer):
    pl = cache.c.page_len
    ids = [int(p) for p in table[b, :-(-n // pl)]]
    k, v = (x[layer, ids].transpose(1, 2).reshape(-1, cache.c.n_kv_heads, cache.c.head_dim)[:n]
            for x in (cache.k, cache.v))
    return k, v


def check(shape, cache, table, lens, q, out, layer, seqs=None):
    for i, b in enumerate(range(len(lens)) if seqs is None else seqs):
        k, v = rows(cache, table, b, lens[b], layer)
        cu.check_attention(out[i:i + 1], cu.attention(q[i:i + 1], k, v, [lens[b]]), shape[0])


@pytest.mark.parametrize("page_len", [16, 48, 128])
@pytest.mark.parametrize("max_len", [0, 2049, 40])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_against_the_definition(shape, page_len, max_len):
    """max_len: unknown (planned from the table), exact, far below the lengths."""
    torch = cu.torch_mod()
    cache, q, table = make(shape, LENS, page_len, extra=7)
    out = torch.full_like(q, 7.0)
    cache.attend(1, q, cu.ints(np.arange(len(LENS))), out, max_len=max_len)
    check(shape, cache, table, LENS, q, out, 1)
    assert not out[0].any()


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[4], SHAPES[5]], ids=str)
def test_one_row_long_context(shape):
    torch = cu.torch_mod()
    lens = [20011]
    cache, q, table = make(shape, lens, 16, layers=1)
    out = torch.full_like(q, 7.0)
    cache.attend(0, q, cu.ints([0]), out)
    check(shape, cache, table, lens, q, out, 0)


@pytest.mark.parametrize("shape", [SHAPES[1], SHAPES[6]], ids=str)
def test_padded_rows_repeats_and_strides(shape):
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    lens = [300, 5, 70]
    cache, _, table = make(shape, lens)
    seqs = [2, -1, 0, 0, 3, 1, 65536]
    wide = cu.randn(dtype, 9, len(seqs), H * D + 64)
    q = wide[:, :H * D].unflatten(1, (H, D))
    full = torch.full((len(seqs), H * D + 32), 7.0, dtype=q.dtype, device="cuda")
    out = full[:, :H * D].unflatten(1, (H, D))
    cache.attend(0, q, cu.ints(seqs), out)
    for i, b in enumerate(seqs):
        if 0 <= b < 3:
            check(shape, cache, table, lens, q[i:i + 1], out[i:i + 1], 0, [b])
        else:
            assert (out[i] == 7).all()
    assert (full[:, H * D:] == 7).all()


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[2], SHAPES[7]], ids=str)
def test_entries_that_are_no_page_hold_no_keys(shape):
    torch = cu.torch_mod()
    lens = [200, 100, 64, 40]
    cache, q, table = make(shape, lens)
    holes = {0: [3, 7], 1: [0], 2: [0, 1, 2, 3], 3: [1, 2]}
    for b, cols in holes.items():
        for j, c in enumerate(cols):
            cache.table[b, c] = (-1, 1 << 20, -(1 << 31), cache.c.n_pages)[j % 4]
    out = torch.full_like(q, 7.0)
    cache.attend(0, q, cu.ints(np.arange(4)), out)
    for b, cols in holes.items():
        k, v = rows(cache, table, b, lens[b], 0)
        keep = [i for i in range(lens[b]) if i // 16 not in cols]
        ref = cu.attention(q[b:b + 1], k[keep], v[keep], [len(keep)])
        cu.check_attention(out[b:b + 1], ref, shape[0])
    assert not out[2].any()
    cache.length.fill_(1 << 30)  # longer than the table: what the table holds
    cache.length[0] = -5
    cache.attend(0, q, cu.ints(np.arange(4)), out)
    assert not out[0].any()


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[5]], ids=str)
def test_scores_that_are_not_finite(shape):
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    lens = [400, 400, 400, 400]
    cache, q, table = make(shape, lens, layers=1)
    q[:, :, 0] = 1.0
    for b, (lo, hi, x) in enumerate([(0, 200, -np.inf), (0, 400, -np.inf), (5, 6, np.nan),
                                     (399, 400, np.inf)]):
        for i in range(lo, hi):
            cache.k[0, table[b, i // 16], :, i % 16, 0] = x
    out = torch.full_like(q, 7.0)
    cache.attend(0, q, cu.ints(np.arange(4)), out)
    k, v = rows(cache, table, 0, 400, 0)
    cu.check_attention(out[:1], cu.attention(q[:1], k[200:], v[200:], [200]), dtype)
    assert out[1:].isnan().all()


def test_offsets_past_32_bits():
    """Pages behind 2^31 elements (2^32 bytes) of a layer, in the second layer."""
    from paper_2608_27384_amd.flashvla import PageCache
    torch = cu.torch_mod()
    D, pl, pages = 256, 256, 36000
    shape = (2, pages, 1, pl, D)
    k, v = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ids = [pages - 1, 5, pages - 7]
    for i, p in enumerate(ids):
        k[1, p] = cu.randn("bf16", 10 + i, 1, pl, D)
        v[1, p] = cu.randn("bf16", 20 + i, 1, pl, D)
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    cache = PageCache(k, v, cu.ints([ids]), cu.ints([700]), refs)
    q = cu.randn("bf16", 30, 1, 8, D)
    out = torch.empty_like(q)
    cache.attend(1, q, cu.ints([0]), out)
    kk, vv = (x[1, ids].reshape(-1, 1, D)[:700] for x in (k, v))
    cu.check_attention(out, cu.attention(q, kk, vv, [700]), "bf16")
    # and an append there
    kn, vn = cu.randn("bf16", 31, 1, 1, D), cu.randn("bf16", 32, 1, 1, D)
    cache.append(1, q.clone(), kn, vn, cu.ints([[0]]), cu.ints([0]), cu.ints([5]), [D // 2])
    assert torch.equal(k[1, ids[0], 0, 5], kn[0, 0]) and torch.equal(v[1, ids[0], 0, 5], vn[0, 0])


def test_two_graphs_and_growing_lengths():
    """Two captured calls replayed on two streams at once keep workspaces of their own, and
    follow the lengths that the cache holds when they run."""
    torch = cu.torch_mod()
    shape = SHAPES[1]
    lens = [1500, 900]
    cache, q, table = make(shape, lens)
    seqs = cu.ints([0, 1])
    outs, graphs = [], []
    for layer in (0, 1):
        out = torch.zeros_like(q)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cache.attend(layer, q, seqs, out, max_len=1500)
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
        for layer in (0, 1):
            check(shape, cache, table, now, q, outs[layer], layer)
            eager = torch.zeros_like(q)
            cache.attend(layer, q, seqs, eager, max_len=1500)
            assert torch.equal(eager, outs[layer])


def test_a_row_does_not_depend_on_the_others():
    torch = cu.torch_mod()
    shape = SHAPES[0]
    cache, q, table = make(shape, [800, 40, 333])
    a, b = torch.zeros_like(q), torch.zeros_like(q)
    cache.attend(0, q, cu.ints([0, 1, 2]), a)
    cache.length[0] = 3
    cache.attend(0, q, cu.ints([0, 1, 2]), b)
    assert torch.equal(a[1:], b[1:]) and not torch.equal(a[0], b[0])


@pytest.mark.parametrize("shape", [(t, 4, 4, D) for t in ("bf16", "fp32") for D in (64, 128, 192, 256)],
                         ids=str)
def test_more_than_the_caches_hold(shape):
    """A layer of more than half a gigabyte, and rows that might read as much: streamed."""
    torch = cu.torch_mod()
    from paper_2608_27384_amd.flashvla import PageCache
    small, q, table = make(shape, LENS, layers=1)
    key = 2 * shape[2] * shape[3] * q.element_size()
    pages = (1 << 29) // (16 * key) + 7
    k, v = (torch.full((1, pages, *x.shape[2:]), float("nan"), dtype=x.dtype, device="cuda")
            for x in (small.k, small.v))
    k[:, :small.k.shape[1]], v[:, :small.v.shape[1]] = small.k, small.v
    wide = np.full((len(LENS), pages), -1)
    wide[:, :table.shape[1]] = table
    refs = np.zeros(pages)
    refs[table[table >= 0]] = 1
    cache = PageCache(k, v, cu.ints(wide), cu.ints(LENS), cu.ints(refs))
    for max_len in (0, pages * 16):
        out = torch.full_like(q, 7.0)
        cache.attend(0, q, cu.ints(range(len(LENS))), out, max_len=max_len)
        check(shape, cache, table, LENS, q, out, 0)


@pytest.mark.parametrize("max_len", [0, 2049])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_probabilities_keep_their_bits(shape, max_len):
    """bf16 values meet probabilities of 16 bits, not of 8."""
    torch = cu.torch_mod()
    cache, q, table = make(shape, LENS)
    out = torch.full_like(q, 7.0)
    cache.attend(1, q, cu.ints(np.arange(len(LENS))), out, max_len=max_len)
    for i, n in enumerate(LENS):
        k, v = rows(cache, table, i, n, 1)
        cu.check_attention_wide(out[i:i + 1], cu.attention(q[i:i + 1], k, v, [n]), shape[0])


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[2], SHAPES[5]], ids=str)
def test_values_that_are_not_finite(shape, bad):
    """An infinite value of a key that is seen gives that infinity, whatever bits its probability
    has: all alike (scores of zero) or spread."""
    torch = cu.torch_mod()
    lens = [1, 40, 700, 2049]
    for zero in (True, False):
        cache, q, table = make(shape, lens, layers=1)
        if zero:
            q.zero_()
        for b, n in enumerate(lens):
            for at, d in ((0, 3), (n - 1, 5), (n // 2, 7)):
                cache.v[0, table[b, at // 16], :, at % 16, d] = bad
        out = torch.full_like(q, 7.0)
        cache.attend(0, q, cu.ints(range(len(lens))), out)
        hit = torch.zeros(shape[3], dtype=torch.bool, device="cuda")
        hit[[3, 5, 7]] = True
        got = out[..., hit]
        assert (got.isnan() if np.isnan(bad) else got == bad).all()
        assert out[..., ~hit].isfinite().all()


@pytest.mark.parametrize("max_len", [0, 4900, 40])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_every_key_counts_once(shape, max_len):
    """With queries of zero every probability is one, and the value of position p in kv head g a one
    at element p + g: a row's result is, times its length, how many positions fall on each element.
    Ones are 1 + 2^-23 in bf16, whose sums of 77 and, for the denominator, of a lane's 20 by 64 lanes
    and 39 chunks, each addition off by 2^-24, stay within 2^-16; with the result's own rounding
    (2^-8) that leaves less than half a key where an element has at most 77."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    lens = [1, 16, 127, 128, 129, 1000, 2048, 3333, 4900]
    cache, q, table = make(shape, lens, 48, layers=1)
    q.zero_()
    cache.v.masked_fill_(~cache.v.isnan(), 0.0)
    g = torch.arange(G, device="cuda")[:, None]
    for b, n in enumerate(lens):
        for j in range(-(-n // 48)):
            p = torch.arange(48 * j, min(48 * j + 48, n), device="cuda")[None]
            cache.v[0, table[b, j], :, :p.shape[1]].scatter_(2, ((p + g) % D)[..., None], 1.0)
    out = torch.full_like(q, 7.0)
    cache.attend(0, q, cu.ints(range(len(lens))), out, max_len=max_len)
    n = torch.tensor(lens, device="cuda")[:, None, None]
    d, h = torch.arange(D, device="cuda")[None, None], (torch.arange(H, device="cuda") * G // H)[None, :, None]
    want = torch.div(n - (d - h) % D + D - 1, D, rounding_mode="floor").clamp(min=0)
    assert int(want.max()) <= 77
    assert bool(((out.double() * n - want).abs() <= want * (cu.EPS[dtype] + 2.0 ** -16)).all())


@pytest.mark.parametrize("page_len", range(16, 257, 16))
@pytest.mark.parametrize("shape", [SHAPES[2], SHAPES[5]], ids=str)
def test_every_page_length(shape, page_len):
    torch = cu.torch_mod()
    lens = [0, 1, page_len - 1, page_len, page_len + 1, 3 * page_len + 17, 16 * page_len, 4000 + page_len]
    cache, q, table = make(shape, lens, page_len, extra=2)
    for max_len in (0, 100):
        out = torch.full_like(q, 7.0)
        cache.attend(1, q, cu.ints(range(len(lens))), out, max_len=max_len)
        check(shape, cache, table, lens, q, out, 1)


@pytest.mark.parametrize("max_len", [0, 1 << 20])
def test_longest_row_of_a_table(max_len):
    """65536 pages of 256 rows, sixteen pages each named 4096 times: the result over every key once.
    Of a chunk's 2048 keys a lane adds 128, and of 8192 chunks a wave 1024, a shorter chain of additions
    than the 4096 of the definition's bound; planned for 2^20 keys the last chunk has the other 2^24,
    of which a lane adds one in 16 (four waves, tiles of 32 keys of which a lane has 8)."""
    from paper_2608_27384_amd.flashvla import PageCache
    torch = cu.torch_mod()
    shape = ("bf16", 8, 1, 64)
    pl, pages, width = 256, 16, 65536
    k, v = (cu.randn("bf16", i, 1, pages, 1, pl, 64) for i in (1, 2))
    ids = np.random.default_rng(0).permutation(np.repeat(np.arange(pages), width // pages))
    n = width * pl
    cache = PageCache(k, v, cu.ints([ids]), cu.ints([n]), cu.ints([width // pages] * pages))
    q = cu.randn("bf16", 3, 1, 8, 64)
    out = torch.full_like(q, 7.0)
    cache.attend(0, q, cu.ints([0]), out, max_len=max_len)
    want, size, soft = cu.attention(q, k[0].reshape(-1, 1, 64), v[0].reshape(-1, 1, 64), [pages * pl])
    if max_len:
        soft = soft + size * (n // 16 * 2.0 ** -24)
    cu.check_attention_wide(out, (want, size, soft), "bf16")
    cache.length.fill_(n - 1)  # one key fewer moves nothing by more than its weight
    again = torch.full_like(q, 7.0)
    cache.attend(0, q, cu.ints([0]), again, max_len=max_len)
    cu.check_attention_wide(again, (want, size, soft + size * 2.0 ** -8), "bf16")


@pytest.mark.parametrize("max_len", [0, 700, 40])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_calls_repeat_themselves(shape, max_len):
    """More workgroups than CUs, in chunks and in one: the same bits from every call."""
    torch = cu.torch_mod()
    lens = [1 + 37 * b % 700 for b in range(300)]
    cache, q, _ = make(shape, lens, layers=1)
    seqs, calls = cu.ints(range(len(lens))), []
    for _ in range(4):
        out = torch.full_like(q, 7.0)
        cache.attend(0, q, seqs, out, max_len=max_len)
        calls.append(out)
    for out in calls:
        assert out.isfinite().all() and out.equal(calls[0])
