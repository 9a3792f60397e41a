"""The cache in 8 bits: what the append writes against the definition in 64 bits, reading back,
the upkeep against a plain model, and the whole path as it is used."""
import random

import numpy as np
import pytest

import context_util as cu
import quant_util as qu
from test_quant_refusals import part_plan

pytestmark = pytest.mark.gpu


def fresh(n_pages, max_seqs, max_pages, page_len=16, layers=2, heads=2, D=64, dtype="bf16", seed=0):
    from paper_2608_27384_amd.flashvla import QuantCache
    cache = QuantCache.empty(layers, heads, D, n_pages, max_seqs, max_pages, page_len, cu.ttype(dtype))
    return qu.fill(cache, seed), cu.Model(n_pages, max_seqs, max_pages, page_len)


def pools(cache):
    torch = cu.torch_mod()
    return [x.view(torch.uint8) for x in cache.pools]


def copies(cache):
    return [x.clone() for x in pools(cache)]


def scattered(cache, lens, seed=0):
    """The table's rows with pages for `lens` positions, all over the pool."""
    pl = cache.c.page_len
    ids = iter(np.random.default_rng(seed).permutation(cache.c.n_pages))
    table = np.full(tuple(cache.table.shape), -1)
    for b, n in enumerate(lens):
        for j in range(-(-n // pl)):
            table[b, j] = next(ids)
    cache.table.copy_(cu.ints(table))
    return table


SHAPES = [("bf16", 8, 1, 256), ("bf16", 4, 2, 64), ("fp32", 3, 1, 192), ("bf16", 8, 8, 128),
          ("fp32", 4, 2, 128), ("bf16", 6, 2, 192), ("fp32", 2, 2, 64), ("fp32", 2, 1, 256), ("bf16", 40, 40, 64)]
IDS = dict(ids=lambda s: "x".join(map(str, s)))


def append(cache, layer, q, k, v, seqs, at, pos=None, sections=None, **kw):
    """Without positions nothing turns: the keys that are quantised are the caller's, exactly."""
    D = q.shape[-1]
    pos = np.zeros((1, len(seqs))) if pos is None else pos
    torch = cu.torch_mod()
    kw.setdefault("q_out", torch.empty_like(q))
    cache.append(layer, q, k, v, cu.ints(pos), cu.ints(seqs), cu.ints(at), sections or (D // 2,), **kw)


class Pair:
    """Keys and values of a layer by the definition, beside the cache's."""

    def __init__(self, cache, layer):
        self.cache, self.layer = cache, layer
        c = cache
        self.k = qu.Written(c.k[layer], c.k_scale[layer], False)
        self.v = qu.Written(c.v[layer], c.v_scale[layer], True)

    def append(self, k, v, seqs, at, table):
        for w, x in ((self.k, k), (self.v, v)):
            w.append(x.double(), list(map(int, seqs)), list(map(int, at)), table, self.cache.c.max_seqs)

    def check(self):
        c, l = self.cache, self.layer
        assert self.k.same(c.k[l], c.k_scale[l], False)
        assert self.v.same(c.v[l], c.v_scale[l], True)


@pytest.mark.parametrize("page_len", [16, 48, 256])
@pytest.mark.parametrize("shape", SHAPES, **IDS)
def test_appended_part_by_part(shape, page_len):
    """Prompts, parts that begin and end inside blocks, single tokens, blocks whose scale grows and
    shrinks on the way; places that do not exist among them; the other layer stays."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    cache, _ = fresh(40 if page_len < 100 else 12, 4, 9 if page_len < 100 else 3, page_len, heads=G, D=D, dtype=dtype)
    holds = cache.c.max_pages * page_len
    table = scattered(cache, [130, 0, 100, 20])
    table[2, 90 // page_len] = -1  # a hole: tokens there are not stored
    cache.table.copy_(cu.ints(table))
    other = copies(cache)
    pair = Pair(cache, 1)
    have = [0, 0, 0, 0]
    for step, (parts, size) in enumerate([((37, 0, 5, 1), 1.0), ((1, 0, 1, 1), 30.0), ((1, 0, 1, 1), 0.01),
                                          ((16, 0, 11, 0), 1e-3), ((3, 0, 70, 14), 4.0), ((60, 0, 13, 1), 500.0)]):
        seqs = np.repeat(range(4), parts)
        at = np.concatenate([have[b] + np.arange(n) for b, n in enumerate(parts)])
        have = [a + b for a, b in zip(have, parts)]
        extra = [(-1, 3), (4, 3), (0, -1), (0, holds), (1, 5), (1 << 30, 1 << 30)]
        seqs, at = np.append(seqs, [s for s, _ in extra]), np.append(at, [p for _, p in extra])
        n = len(seqs)
        q, k, v = (cu.randn(dtype, 10 * step + i, n, h, D, std=size) for i, h in enumerate((H, G, G)))
        ko = torch.full_like(k, 7.0)
        append(cache, 1, q, k, v, seqs, at, k_out=ko if step % 2 else None)
        pair.append(k, v, seqs, at, table)
        pair.check()
        if step % 2:
            assert ko.equal(k)
    for x, y in zip(pools(cache), other):
        assert x[0].equal(y[0])


@pytest.mark.parametrize("n", [1, 17, 127, 128, 1023, 1024, 4099, 8197])
@pytest.mark.parametrize("shape", SHAPES[:6], **IDS)
def test_rotated_and_quantised(shape, n):
    """Keys are off by half a step of e4m3 and the rotation's own error; scales are those of the
    largest, queries and kept keys the rotary operator's.  Runs of tokens lie in both sequences, from
    position 5 on, and cross what workgroups share out, 1, 4 or 8 tokens of the list,
    and the shares of workgroups that have the same tokens."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    rng = np.random.default_rng(n)
    sections = (D // 8, 3 * D // 16, 3 * D // 16)
    lens = [n // 3, n - n // 3]
    cache, _ = fresh(n // 16 + 8, 3, n // 16 + 3, 16, heads=G, D=D, dtype=dtype)
    table = scattered(cache, [lens[0] + 5, 0, lens[1] + 5])
    seqs = np.repeat([0, 2], lens)
    at = np.concatenate([5 + np.arange(x) for x in lens])
    pos = rng.integers(-50, 4000, (3, n))
    pos[0, 0], pos[-1, n // 2] = 1 << 24, -(1 << 20)
    qkv = cu.randn(dtype, n, n, H + 2 * G, D)
    q, k, v = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
    qo, ko = (torch.zeros(n, h, D, dtype=q.dtype, device="cuda") for h in (H, G))
    ref_v = qu.Written(cache.v[1], cache.v_scale[1], True)
    before = qu.exponents(cache.k_scale[1])
    append(cache, 1, q, k, v, seqs, at, pos, sections, q_out=qo, k_out=ko, theta=5e5)
    far = float(np.abs(pos).max()) * 2.0 ** -50
    cu.check_rotated(qo, cu.rotate(q, pos, sections, 5e5), dtype, far)
    want, size, whole = cu.rotate(k, pos, sections, 5e5)
    cu.check_rotated(ko, (want, size, whole), dtype, far)
    ref_v.append(v.double(), seqs.tolist(), at.tolist(), table, 3)
    assert ref_v.same(cache.v[1], cache.v_scale[1], True)
    off = 3 * 2.0 ** -24 * size + whole * (2.0 ** -21 + far)
    page = torch.from_numpy(table[seqs, at // 16]).cuda()
    e = qu.exponents(cache.k_scale[1])
    for i, j in qu.runs(seqs.tolist(), at.tolist(), 1 << 30, 3):
        lo, hi = (qu.exponent_for((want[i:j].abs() + s * off[i:j]).clamp(min=0).amax((0, 2))) for s in (-1, 1))
        p = int(page[i])
        if at[i] % 16:
            lo, hi = torch.maximum(lo, before[p, :, 0]), torch.maximum(hi, before[p, :, 0])
        assert bool(((e[p, :, 0] >= lo) & (e[p, :, 0] <= hi)).all()), (i, j)
    rows = torch.from_numpy(at % 16).cuda()
    got = qu.decoded(cache.k[1], cache.k_scale[1], False)[page, :, rows]
    unit = torch.exp2(e[page, :, 0].double())[..., None]
    tol = off + torch.maximum(2.0 ** -10 * unit, 2.0 ** -4 * (want.abs() + off))
    assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() - tol).max())


@pytest.mark.parametrize("D", [64, 128, 192, 256])
def test_turned_as_64_bits_turn(D):
    """Cosines and sines are off by half a step of fp32 at one (2^-25) and 2^-33, products and the sum
    by another 2^-24 each of a result of |a| + |b| at most; the positions' turns in 64 bits by
    2^-50 of them.  Every eighth of a turn is among the angles."""
    torch = cu.torch_mod()
    n = 4096
    cache, _ = fresh(4, 1, 1, 16, heads=1, D=D, dtype="fp32")
    q, k = cu.randn("fp32", D, n, 2, D), cu.randn("fp32", D + 1, n, 1, D)
    pos = np.concatenate([np.arange(-1024, 1024), np.random.default_rng(D).integers(-1 << 20, 1 << 20, 2048)])[None]
    for theta in (1e4, 2.0 * np.pi):
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        append(cache, 0, q, k, k, np.full(n, -1), np.zeros(n), pos, theta=theta, q_out=qo, k_out=ko)
        for got, x in ((qo, q), (ko, k)):
            want, _, whole = cu.rotate(x, pos, (D // 2,), theta)
            tol = (2.5 * 2.0 ** -24 + 2.0 ** -33 + (1 << 20) * 2.0 ** -50) * (1 + 2.0 ** -20)
            assert bool(((got.double() - want).abs() <= tol * whole).all()), float(((got.double() - want).abs() / whole).max())


def test_a_block_starts_anew_and_goes_on():
    """From its first position on: zeros behind the new ones and a scale of theirs alone.  From
    another: the scale does not fall, the rows on both sides stay, gaps are left as they are."""
    torch = cu.torch_mod()
    H, G, D = 2, 2, 64
    cache, _ = fresh(4, 2, 2, 32, layers=1, heads=G, D=D)
    table = scattered(cache, [64, 64])
    pair = Pair(cache, 0)
    for step, (at, size) in enumerate([([0, 1, 5], 100.0), ([9], 1.0), ([2, 3], 1e4), ([4, 6, 7, 15], 1e-4),
                                       ([16], 1e-6), ([17, 31], 1e6), ([0], 1.0), ([15], 3.0), ([33], 2.0)]):
        n = len(at)
        q, k, v = (cu.randn("bf16", 3 * step + i, n, h, D, std=size) for i, h in enumerate((H, G, G)))
        append(cache, 0, q, k, v, [1] * n, at)
        pair.append(k, v, [1] * n, at, table)
        pair.check()
        page = table[1, 0]
        if step == 0:
            codes = qu.rows_of(cache.v[0], True)[page]
            assert not codes[:, [2, 3, 4] + list(range(6, 16))].any() and codes[:, [0, 1, 5]].any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rounding_at_every_border(dtype):
    """Every number of e4m3, every middle between two and its neighbours in the type, at scales of
    2^-117, 1 and 2^119, both signs; a block's largest sets the scale."""
    torch = cu.torch_mod()
    D = 64
    pos = torch.from_numpy(qu.NUMBERS[:127])
    mids = (pos[:-1] + pos[1:]) / 2
    near = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -23
    x = torch.cat([pos, mids, mids * (1 + near), mids * (1 - near)])
    x = torch.cat([x, -x])
    x = x[:len(x) // (D - 1) * (D - 1)].reshape(-1, D - 1)
    x = torch.cat([x, torch.full((len(x), 1), 448.0)], 1)
    for e in (-117, 0, 119):
        y = (x * 2.0 ** e).to(cu.ttype(dtype)).cuda()[:, None]  # a token a block
        n = len(y)
        cache, _ = fresh(n, n, 1, 16, layers=1, heads=1, D=D, dtype=dtype)
        table = scattered(cache, [16] * n)
        pair = Pair(cache, 0)
        append(cache, 0, y, y, y, range(n), [0] * n)
        pair.append(y, y, range(n), [0] * n, table)
        pair.check()
        used = torch.from_numpy(table[:, 0]).cuda()
        assert bool((qu.exponents(cache.k_scale[0])[used] == e).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_extreme_values(dtype):
    """Zeros, infinities, NaN, the type's largest and smallest: what is not finite is NaN and does
    not set the scale, what is past 448 of the largest scale saturates."""
    torch = cu.torch_mod()
    D, t = 64, cu.ttype(dtype)
    big, tiny = torch.finfo(t).max, torch.finfo(t).tiny
    rows = [[0.0], [np.inf, 1.0], [-np.inf, np.nan, 2.0], [np.nan], [big, -big, 1.0], [tiny, -tiny], [tiny / 64],
            [big, tiny], [1.75 * 2.0 ** 127, -1.0], [448.0], [448.0 * (1 + 2.0 ** -7)], [1.0, 2.0 ** -20]]
    x = torch.tensor([(r * D)[:D] for r in rows], dtype=torch.float64).to(t).cuda()[:, None]
    n = len(rows)
    for at in (0, 7):  # anew, and over what a block holds
        cache, _ = fresh(n, n, 1, 16, layers=1, heads=1, D=D, dtype=dtype)
        table = scattered(cache, [16] * n)
        pair = Pair(cache, 0)
        append(cache, 0, x, x, x, range(n), [at] * n)
        for w in (pair.k, pair.v):
            w.append(x.double(), list(range(n)), [at] * n, table, n)
        c = cache
        assert pair.v.same(c.v[0], c.v_scale[0], True)
        # keys turn by nothing: inf * 0 is NaN, in the pair's other half too
        fine = torch.tensor([bool(np.isfinite(r).all()) for r in rows])
        used = torch.from_numpy(table[:, 0])[fine].cuda()
        a = qu.numbers(qu.rows_of(c.k[0], False))[used]
        assert a.equal(qu.numbers(pair.k.codes)[used])
        assert qu.exponents(c.k_scale[0])[used].equal(pair.k.e[used])
        odd = torch.from_numpy(table[:, 0])[~fine].cuda()
        assert qu.numbers(qu.rows_of(c.k[0], False))[odd][:, :, at].isnan().any(-1).all()


def test_a_token_of_another_list_order():
    """Blocks listed in any order, sequences mixed, as long as a block's tokens stand together."""
    torch = cu.torch_mod()
    H, G, D = 2, 2, 128
    rng = np.random.default_rng(0)
    cache, _ = fresh(200, 5, 40, 16, layers=1, heads=G, D=D)
    table = scattered(cache, [500, 640, 33, 200, 17])
    parts = [(s, b) for s, n in enumerate([500, 640, 33, 200, 17]) for b in range(-(-n // 16))]
    seqs, at = [], []
    for i in rng.permutation(len(parts)):
        s, b = parts[i]
        rows = sorted(rng.choice(16, rng.integers(1, 17), replace=False))
        seqs += [s] * len(rows)
        at += [16 * b + int(r) for r in rows]
    for lo, hi in ((0, 700), (0, len(seqs))):  # few tokens a workgroup, and many by repeating the list
        sq, p = seqs[lo:hi], at[lo:hi]
        k, v = (cu.randn("bf16", i, len(sq), G, D) for i in (1, 2))
        pair = Pair(cache, 0)
        append(cache, 0, cu.randn("bf16", 3, len(sq), H, D), k, v, sq, p)
        pair.append(k, v, sq, p, table)
        pair.check()
    # more than 2048 tokens, the list twice: the second time over what the first wrote
    other, _ = fresh(200, 5, 40, 16, layers=1, heads=G, D=D, seed=4)
    other.table.copy_(cache.table)
    reps = -(-2100 // len(seqs))
    pair = Pair(other, 0)
    assert len(seqs) * reps >= 2048
    far = [s for _ in range(reps) for s in seqs]
    # one repetition has places, the others pad the list
    far = [s if i < len(seqs) else -1 for i, s in enumerate(far)]
    p = at * reps
    k, v = (cu.randn("bf16", i, len(far), G, D) for i in (5, 6))
    append(other, 0, cu.randn("bf16", 7, len(far), H, D), k, v, far, p)
    pair.append(k, v, far, p, table)
    pair.check()


def test_places_named_twice_touch_nothing_else():
    torch = cu.torch_mod()
    D = 64
    cache, _ = fresh(10, 2, 4, 16, layers=1, heads=1, D=D)
    table = scattered(cache, [64, 64])
    before = copies(cache)
    seqs, at = [0] * 40, [3, 3, 2, 5] * 10
    k = cu.randn("bf16", 1, 40, 1, D)
    ko = torch.zeros_like(k)
    append(cache, 0, k, k, k, seqs, at, k_out=ko)
    assert ko.equal(k)
    for x, y in zip(pools(cache), before):
        x = x.clone()
        x[:, table[0, 0]] = y[:, table[0, 0]]
        assert x.equal(y)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_in_place_strided_and_on_another_stream(dtype):
    torch = cu.torch_mod()
    H, G, D, n = 4, 2, 64, 37
    cache, _ = fresh(12, 2, 4, 16, heads=G, D=D, dtype=dtype)
    scattered(cache, [64, 64])
    seqs, at = [0] * 20 + [1] * 17, list(range(3, 23)) + list(range(17))
    pos = np.arange(n)[None]
    packed = cu.randn(dtype, 5, n, H + 2 * G, D)
    q, k, v = packed[:, :H], packed[:, H:H + G], packed[:, H + G:]
    qo, ko = (torch.empty(n, h, D, dtype=q.dtype, device="cuda") for h in (H, G))
    start = copies(cache)
    append(cache, 1, q, k, v, seqs, at, pos, q_out=qo, k_out=ko)
    want, clean = copies(cache), v.clone()
    for x, y in zip(pools(cache), start):
        x.copy_(y)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    args = [cu.ints(x) for x in (pos, seqs, at)]
    torch.cuda.synchronize()
    cache.append(1, q, k, v, *args, (D // 2,), k_out=k, stream=s)
    s.synchronize()
    assert q.equal(qo) and k.equal(ko) and v.equal(clean)
    assert all(x.equal(y) for x, y in zip(pools(cache), want))


def test_nothing_to_append():
    torch = cu.torch_mod()
    cache, _ = fresh(4, 2, 2)
    before = copies(cache)
    q, k = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    append(cache, 0, q, k, k, [], [])
    assert all(x.equal(y) for x, y in zip(pools(cache), before))


def test_offsets_past_32_bits():
    """Codes behind 2^32 bytes of a layer, in the second layer: written, read back, attended to."""
    from paper_2608_27384_amd.flashvla import QuantCache
    torch = cu.torch_mod()
    D, pl, pages = 256, 256, 66000
    cache = QuantCache.empty(2, 1, D, pages, 1, 3, pl)
    cache.k.view(torch.uint8).zero_()
    cache.v.view(torch.uint8).zero_()
    cache.k_scale.view(torch.uint8).fill_(120)
    cache.v_scale.view(torch.uint8).fill_(120)
    ids = [pages - 1, 5, pages - 7]
    cache.table.copy_(cu.ints([ids]))
    n = 700
    cache.length.copy_(cu.ints([n]))
    q, k, v = (cu.randn("bf16", i, n, h, D) for i, h in enumerate((8, 1, 1)))
    append(cache, 1, q, k, v, [0] * n, range(n))
    kd, vd = (torch.empty(2, 1, n, 1, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache.gather(cu.ints([0]), kd, vd)
    for got, x in ((kd, k), (vd, v)):
        assert not got[0].any()
        blocks = torch.nn.functional.pad(x.double().abs().amax((1, 2)), (0, 4)).view(-1, 16).amax(1)
        unit = torch.exp2(qu.exponent_for(blocks).double()).repeat_interleave(16)[:n, None, None]
        err = (got[1, 0].double() - x.double()).abs()
        assert bool((err <= torch.maximum(2.0 ** -10 * unit, 2.0 ** -4 * x.double().abs())).all())
    out = torch.empty(1, 8, D, dtype=torch.bfloat16, device="cuda")
    cache.attend(1, q[-1:], cu.ints([0]), out)
    ref = qu.attention(q[-1:], kd[1, 0].double(), vd[1, 0].double(), [n], "bf16")
    cu.check_attention_wide(out, ref, "bf16")
    cache.attend_part(1, q[-1:], cu.ints([0, 1]), cu.ints([0]), out)
    cu.check_attention(out, ref, "bf16")
    ref = qu.attention(q, kd[1, 0].double(), vd[1, 0].double(), range(1, n + 1), "bf16")
    for times, rows in ((3, 64), (20, 128)):  # of the whole sequence
        assert part_plan(times * n, times, 8, 1, D, 3 * pl).rows == rows
        out = torch.empty(times * n, 8, D, dtype=torch.bfloat16, device="cuda")
        cache.attend_part(1, q.repeat(times, 1, 1), cu.ints(n * np.arange(times + 1)), cu.ints([0] * times), out)
        for i in range(times):
            cu.check_attention(out[n * i:n * (i + 1)], ref, "bf16")


# ------------------------------------------------------------------ reading back

@pytest.mark.parametrize("page_len", [16, 48, 256])
@pytest.mark.parametrize("shape", SHAPES, **IDS)
def test_read_back(shape, page_len):
    """Exactly what the codes stand for; rows past a length, holes and entries without a sequence
    stay; codes of every kind, NaN among them, at scales from 2^-117 to 2^119."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    cache, _ = fresh(60, 6, 9, page_len, layers=3, heads=G, D=D, dtype=dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for x in pools(cache)[:2]:
        x.copy_(torch.randint(0, 256, x.shape, generator=g, device="cuda").to(torch.uint8))
    for x in pools(cache)[2:]:
        x.copy_(torch.randint(10, 247, x.shape, generator=g, device="cuda").to(torch.uint8))
    lens = [1, page_len + 1, 3 * page_len + 5, 0, 7 * page_len - 1, 2]
    table = scattered(cache, lens)
    table[2, 1] = -1
    table[4, 2] = 60
    cache.table.copy_(cu.ints(table))
    cache.length.copy_(cu.ints(lens))
    seqs, ld = [4, 0, 2, -1, 2, 3, 6, 1], 5 * page_len + 3
    k, v = (cu.randn(dtype, i, 3, len(seqs), ld, G, D) for i in (7, 8))
    want = [k.clone(), v.clone()]
    for w, pool, scale, values in ((want[0], cache.k, cache.k_scale, False), (want[1], cache.v, cache.v_scale, True)):
        x = qu.decoded(pool, scale, values).to(w.dtype).transpose(2, 3)
        for i, s in enumerate(seqs):
            for j in range(-(-min(lens[s], ld) // page_len) if 0 <= s < 6 else 0):
                n, p = min(lens[s], ld, (j + 1) * page_len) - j * page_len, table[s, j]
                if 0 <= p < 60:
                    w[:, i, j * page_len:j * page_len + n] = x[:, p, :n]
    cache.gather(cu.ints(seqs), k, v)
    for got, w in ((k, want[0]), (v, want[1])):
        assert got.isnan().equal(w.isnan()) and got.nan_to_num(0).equal(w.nan_to_num(0))


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("fp32", 192), ("bf16", 256), ("fp32", 128)])
def test_copies_of_more_than_the_caches_hold(dtype, D):
    """Read back and compacted in a pool of more than half a gigabyte."""
    torch = cu.torch_mod()
    G, L = 2, 4
    pages = (1 << 29) // (16 * 2 * L * G * D) + 9
    cache, model = fresh(pages, 5, pages, layers=L, heads=G, D=D, dtype=dtype)
    lens = [70, (pages // 2) * 16 - 3, 1, 0, pages * 5 + 1]
    assert int(cache.grow(cu.ints(range(5)), cu.ints(lens))) == 0
    model.grow(list(range(5)), lens)

    def gathered(seqs, ld):
        k, v = (torch.full((L, len(seqs), ld, G, D), 7.0, dtype=cache.dtype, device="cuda") for _ in range(2))
        cache.gather(cu.ints(seqs), k, v)
        return k, v

    ld = lens[1] + 40
    got = gathered([4, 1], ld)
    table = cache.table.long()
    for i, s in enumerate((4, 1)):
        ids = table[s, :-(-lens[s] // 16)]
        for out, pool, scale, values in ((got[0], cache.k, cache.k_scale, False), (got[1], cache.v, cache.v_scale, True)):
            for l in range(L):
                at = torch.arange(0, len(ids), max(1, len(ids) // 300), device="cuda")
                x = qu.decoded(pool.view(torch.uint8)[l, ids[at]].view(torch.float8_e4m3fn),
                               scale.view(torch.uint8)[l, ids[at]].view(torch.float8_e8m0fnu), values)
                want = x.transpose(1, 2).to(cache.dtype)
                rows = (at * 16)[:, None] + torch.arange(16, device="cuda")
                have = rows < lens[s]
                assert out[l, i][rows.clamp(max=ld - 1)][have].equal(want[have])
            assert bool((out[:, i, lens[s]:] == 7).all())
    assert int(cache.free(cu.ints([1]))) == 0
    model.free([1])
    before = gathered([4, 0, 2], ld)
    used, _ = model.compact()
    assert int(cache.compact()) == used
    after = gathered([4, 0, 2], ld)
    assert before[0].equal(after[0]) and before[1].equal(after[1])


# ------------------------------------------------------------------ upkeep

@pytest.mark.parametrize("n_pages,page_len,dtype,D,G", [(60, 16, "bf16", 64, 2), (33, 48, "fp32", 64, 1),
                                                        (20000, 16, "bf16", 64, 1), (90, 32, "bf16", 192, 3)])
def test_random_steps(n_pages, page_len, dtype, D, G):
    """Grown, forked, freed and compacted at random, with lists that fail among them: the pages and
    scales go where the model says, and nothing else changes."""
    seqs, width = 24, 12
    cache, model = fresh(n_pages, seqs, width, page_len, dtype=dtype, D=D, heads=G)
    rng = random.Random(n_pages)
    want = copies(cache)
    seen = set()
    for step in range(120):
        op = rng.choice(["grow", "grow", "grow", "fork", "fork", "free", "compact"])
        n = rng.randint(0, 8)
        pick = lambda: [rng.randint(-1 if rng.random() < 0.02 else 0, seqs - 1) for _ in range(n)]
        some = rng.sample(range(seqs), n)
        if op == "grow":
            add = [rng.choice([0, 1, page_len - 1, page_len, 3 * page_len + 1]) for _ in range(n)]
            got, st = cache.grow(cu.ints(some), cu.ints(add)), model.grow(some, add)
        elif op == "fork":
            empty = [s for s in range(seqs) if model.len[s] == 0]
            kids = rng.sample(empty, min(n, len(empty))) if rng.random() < 0.9 else some
            full = [s for s in range(seqs) if model.len[s]] or [0]
            par = [rng.choice(full) for _ in kids] if rng.random() < 0.9 else pick()[:len(kids)]
            kids = kids[:len(par)]
            got = cache.fork(cu.ints(par), cu.ints(kids))
            st, moved = model.fork(par, kids)
            for a, b, r in moved:
                blocks = -(-r // 16)
                for x in want[:2]:
                    x[:, b, :, :16 * blocks] = x[:, a, :, :16 * blocks]
                for x in want[2:]:
                    x[:, b, :, :blocks] = x[:, a, :, :blocks]
        elif op == "free":
            s = pick()
            got, st = cache.free(cu.ints(s)), model.free(s)
        else:
            got = cache.compact()
            st, moves = model.compact()
            for a, b in moves:
                for x in want:
                    x[:, b] = x[:, a]
        assert int(got) == st, (step, op)
        seen.add((op, st if op != "compact" else 0))
        live = np.arange(width)[None] < -(-model.len // page_len)[:, None]
        assert np.array_equal(cache.length.cpu().numpy(), model.len)
        assert np.array_equal(cache.refs.cpu().numpy(), model.refs)
        assert np.array_equal(cache.table.cpu().numpy()[live], model.table[live])
    assert all(x.equal(y) for x, y in zip(pools(cache), want))
    assert {("grow", 0), ("fork", 0), ("fork", 1), ("free", 0), ("free", 1)} <= seen


def test_written_tensors_move_their_versions():
    torch = cu.torch_mod()
    cache, _ = fresh(20, 4, 4)
    q, k, v = (cu.randn("bf16", i, 5, h, 64) for i, h in enumerate((4, 2, 2)))
    out = torch.empty_like(q)
    at, seqs, st = cu.ints(range(5)), cu.ints([0] * 5), torch.empty(1, dtype=torch.int32, device="cuda")
    kd, vd = (torch.empty(2, 1, 5, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    books, held = [cache.table, cache.length, cache.refs, st], list(cache.pools)
    every = books + held + [q, k, v, out, kd, vd]

    def moved(call, want):
        before = [t._version for t in every]
        call()
        got = {t.data_ptr() for t, b in zip(every, before) if t._version != b}
        assert got == {t.data_ptr() for t in want}

    moved(lambda: cache.grow(cu.ints([0]), cu.ints([5]), st), books)
    moved(lambda: cache.append(0, q, k, v, at[None], seqs, at, (32,)), held + [q])
    moved(lambda: cache.attend(0, q, seqs, out), [out])
    moved(lambda: cache.attend_part(0, q, cu.ints([0, 5]), cu.ints([0]), out), [out])
    moved(lambda: cache.fork(cu.ints([0]), cu.ints([1]), st), books + held)
    moved(lambda: cache.gather(cu.ints([0]), kd, vd), [kd, vd])
    moved(lambda: cache.compact(st), books + held)
    moved(lambda: cache.free(cu.ints([0]), st), books)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_tokens_that_are_taken_back(dtype):
    """Large tokens appended behind five of a block, then left out by a shorter length: the five are
    rounded at the grown scale and stay so.  Appended to a fork they change nothing of the parent's."""
    torch = cu.torch_mod()
    cache, _ = fresh(20, 4, 4, layers=1, dtype=dtype)
    G, D = cache.c.n_kv_heads, cache.c.head_dim

    def append(seq, at, size):
        n = len(at)
        q, k, v = (cu.randn(dtype, 7 + i, n, h, D, std=size) for i, h in enumerate((2 * G, G, G)))
        assert int(cache.grow(cu.ints([seq]), cu.ints([n]))) == 0
        cache.append(0, q, k, v, cu.ints([at]), cu.ints([seq] * n), cu.ints(at), (D // 2,))

    def held(seq):
        kd, vd = (torch.zeros(1, 1, 21, G, D, dtype=cu.ttype(dtype), device="cuda") for _ in range(2))
        cache.gather(cu.ints([seq]), kd, vd)
        return kd, vd

    append(0, range(21), 1.0)
    first = held(0)
    assert int(cache.fork(cu.ints([0]), cu.ints([1]))) == 0
    append(1, range(21, 24), 1e4)
    cache.length[1] = 21
    for seq, same in ((0, True), (1, False)):
        for a, b in zip(held(seq), first):
            assert a[:, :, :16].equal(b[:, :, :16]) and a[:, :, 16:].equal(b[:, :, 16:]) == same


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_context_of_a_run(dtype):
    """Three observations, two layers, in 8 bits: prompts appended and attended to as parts, two more
    tokens each, one by one, a chunk of seven, one sequence forked, one freed, the pool compacted;
    what is read back is what the action expert then decodes against.  Each attention is held to the
    cache's own contents, each of those to the tokens that were appended, by half a step of e4m3 at
    the scale of the largest of the run's values: 4 half steps of 2^-10 of it at most, since a block's
    scale grows at most as often as tokens come in three steps behind its first."""
    import oracle
    import synth
    from gpu_util import Case, host, rel_err, tol
    from paper_2608_27384_amd.flashvla import QuantCache
    torch = cu.torch_mod()
    w = synth.workload("small_bf16_b3").replace(prefix_len=140, dtype=dtype)
    H, G, D, L = w.n_q_heads, w.n_kv_heads, w.head_dim, w.n_layers
    lens, sections = [90, 33, 120], (16, 24, 24)
    cache = QuantCache.empty(L, G, D, 64, 6, 10, 16, cu.ttype(dtype))
    for x in pools(cache):
        x.fill_(255)
    seqs = [0, 1, 2]
    kept = [[[[], []] for _ in seqs] for _ in range(L)]

    def step(new, starts, seed):
        n = sum(new)
        assert int(cache.grow(cu.ints(seqs), cu.ints(new))) == 0
        at = np.concatenate([s + np.arange(x) for s, x in zip(starts, new)])
        edges = np.cumsum([0] + new)
        for l in range(L):
            q, k, v = (cu.randn(dtype, seed + 3 * l + i, n, x, D) for i, x in enumerate((H, G, G)))
            ko = torch.empty_like(k)
            cache.append(l, q, k, v, cu.ints(np.stack([at, at // 4, at % 4])), cu.ints(np.repeat(seqs, new)),
                         cu.ints(at), sections, k_out=ko)
            out = torch.empty_like(q)
            if n > 3:
                cache.attend_part(l, q, cu.ints(edges), cu.ints(seqs), out)
            else:
                cache.attend(l, q, cu.ints(seqs), out)
            table = cache.table.cpu().numpy()
            for b in seqs:
                m = starts[b] + new[b]
                part = slice(edges[b], edges[b + 1])
                kept[l][b][0].append(ko[part].double())
                kept[l][b][1].append(v[part].double())
                kk, vv = qu.context(cache, table, b, m, l)
                for got, want in ((kk, torch.cat(kept[l][b][0])), (vv, torch.cat(kept[l][b][1]))):
                    unit = torch.exp2(qu.exponent_for(want.abs().max()).double())
                    # a kept key was rounded to the dtype, which its code was not
                    size = want.abs() * (2.0 ** -4 + cu.EPS[dtype] * (1 + 2.0 ** -4))
                    assert bool(((got - want).abs() <= torch.maximum(size, 4 * 2.0 ** -10 * unit + size)).all())
                ref = qu.attention(q[part], kk, vv, [starts[b] + i + 1 for i in range(new[b])], dtype)
                cu.check_attention(out[part], ref, dtype)
        return [a + b for a, b in zip(starts, new)]

    now = step(lens, [0, 0, 0], 100)
    now = step([1, 1, 1], now, 200)
    now = step([1, 1, 1], now, 300)
    now = step([7, 7, 7], now, 400)
    assert int(cache.fork(cu.ints([0]), cu.ints([4]))) == 0
    before = {b: [qu.context(cache, cache.table.cpu().numpy(), b, now[b], l) for l in range(L)] for b in seqs}
    assert int(cache.free(cu.ints([0]))) == 0
    cache.compact()
    case = Case(w, lens=[now[1], now[0], now[2]])
    try:
        shape = (L, 3, 140, G, D)
        kd, vd = (torch.full(shape, float("nan"), dtype=cu.ttype(dtype), device="cuda") for _ in range(2))
        cache.gather(cu.ints([1, 4, 2]), kd, vd)
        for i, b in enumerate((1, 0, 2)):
            for l in range(L):
                assert kd[l, i, :now[b]].double().equal(before[b][l][0])
                assert vd[l, i, :now[b]].double().equal(before[b][l][1])
        case.ex.set_prefix(kd, vd, case.lens)
        case.k, case.v = (np.nan_to_num(x.float().cpu().numpy()) for x in (kd, vd))
        new, ref = oracle.decode_step(case.x, case.t, case.k, case.v, case.lens, case.W, w, noise_seed=0, step=0)
        case.ex.decode_step(case.xd, case.td, case.out)
        got = host(case.out)
        for b in range(3):
            assert rel_err(got[b], ref[b]) < tol(w)
    finally:
        case.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_captured_token_step(dtype):
    """A token step of two layers (room, append, attention of the token and of it as a part) in one
    graph, replayed over block and page ends with the eager steps of another cache between."""
    torch = cu.torch_mod()
    H, G, D, L, n = 4, 2, 64, 2, 5
    both = []
    for _ in range(2):
        cache, _ = fresh(60, 6, 8, 32, layers=L, heads=G, D=D, dtype=dtype, seed=3)
        cache.grow(cu.ints(range(6)), cu.ints([1, 15, 16, 0, 31, 40]))
        both.append(cache)
    seqs = cu.ints([4, 0, 2, 1, -1])
    cum = cu.ints(range(n + 1))
    live = seqs.long()[:4]
    x = [cu.randn(dtype, 20 + i, n, h, D) for i, h in enumerate((H, G, G))]

    def buffers():
        return dict(q=torch.empty_like(x[0]), out=[torch.zeros_like(x[0]) for _ in range(2 * L)],
                    at=torch.zeros(n, dtype=torch.int32, device="cuda"),
                    one=torch.ones(4, dtype=torch.int32, device="cuda"), few=seqs[:4].clone(),
                    status=torch.empty(1, dtype=torch.int32, device="cuda"))

    def step(cache, b):
        cache.grow(b["few"], b["one"], b["status"])
        b["at"][:4].copy_(cache.length.index_select(0, live) - 1)
        for l in range(L):
            cache.append(l, x[0], x[1], x[2], b["at"].view(1, n), seqs, b["at"], (D // 2,), q_out=b["q"])
            cache.attend(l, b["q"], seqs, b["out"][2 * l])
            cache.attend_part(l, b["q"], cum, seqs, b["out"][2 * l + 1])

    a, b = buffers(), buffers()
    before = copies(both[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(both[0], a)
    assert all(p.equal(y) for p, y in zip(pools(both[0]), before))
    for i in range(20):
        for t, scale in zip(x, (0.9, 1.1, -0.8)):
            t.mul_(scale)
        g.replay()
        step(both[1], b)
        torch.cuda.synchronize()
        assert a["status"].item() == 0 and b["status"].item() == 0
        assert all(p.equal(y) for p, y in zip(pools(both[0]), pools(both[1])))
        for l in range(2 * L):
            assert a["out"][l].equal(b["out"][l]) and (a["out"][l][4] == 0).all()
    assert both[0].length.tolist() == [21, 35, 36, 0, 51, 40]
