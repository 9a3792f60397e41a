"""Prompt attention against the 64-bit form: packed lengths from zero to several
tiles, keys longer and shorter than the queries, every head dim, grouped heads,
strided rows; what a query does not see has no influence; refusals leave no
trace."""
import numpy as np
import pytest

import context_util as cu

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", 8, 1, 256), ("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("bf16", 6, 2, 192),
          ("bf16", 5, 1, 128), ("fp32", 4, 2, 64), ("fp32", 2, 1, 256), ("fp32", 3, 3, 192),
          ("fp32", 8, 2, 128)]
# Enough rows (300 tokens or so by these heads) for the kernels of fuller chips:
# eight waves halving the keys, four waves, fp32
FULL = [("bf16", 64, 4, D) for D in (64, 128, 192, 256)] + [
    ("bf16", 128, 16, D) for D in (64, 128, 192, 256)] + [("bf16", 126, 18, 128)] + [
    ("fp32", 512, 32, D) for D in (64, 128, 192, 256)]
# (queries, keys) of each prompt
LENS = {"ragged": [(0, 0), (1, 1), (33, 33), (64, 64), (65, 65), (0, 5), (130, 130), (7, 7)],
        "tails": [(1, 300), (5, 64), (32, 97), (3, 3), (100, 517)],
        "empty_rows": [(9, 4), (70, 33), (5, 0), (40, 40), (1, 0)],
        "long": [(700, 700), (31, 950)]}


def make(shape, lens, seed=0):
    dtype, H, G, D = shape
    nq, nk = sum(a for a, _ in lens), sum(b for _, b in lens)
    q, k, v = (cu.randn(dtype, seed + i, n, h, D) for i, (n, h) in
               enumerate(((nq, H), (nk, G), (nk, G))))
    cq = np.cumsum([0] + [a for a, _ in lens])
    ck = np.cumsum([0] + [b for _, b in lens])
    return q, k, v, cq, ck


def run(q, k, v, cq, ck, causal, out=None, **kw):
    from paper_2608_27384_amd.flashvla import prompt_attention
    torch = cu.torch_mod()
    out = torch.full_like(q, 7.0) if out is None else out
    prompt_attention(q, k, v, cu.ints(cq), cu.ints(ck), out, causal=causal, **kw)
    torch.cuda.synchronize()
    return out


def limits(nq, nk, causal):
    return [max(0, min(nk, nk - nq + i + 1)) if causal else nk for i in range(nq)]


def check(shape, out, q, k, v, cq, ck, causal, scale=None):
    for b in range(len(cq) - 1):
        nq, nk = cq[b + 1] - cq[b], ck[b + 1] - ck[b]
        ref = cu.attention(q[cq[b]:cq[b + 1]], k[ck[b]:ck[b + 1]], v[ck[b]:ck[b + 1]],
                           limits(nq, nk, causal), scale)
        cu.check_attention(out[cq[b]:cq[b + 1]], ref, shape[0])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_against_the_definition(shape, lens, causal):
    q, k, v, cq, ck = make(shape, LENS[lens])
    out = run(q, k, v, cq, ck, causal)
    check(shape, out, q, k, v, cq, ck, causal)
    if lens == "empty_rows":
        assert not out[cq[2]:cq[3]].any() and not out[cq[4]:].any()
        if causal:
            assert not out[:5].any()


@pytest.mark.parametrize("lens,causal", [("ragged", True), ("ragged", False), ("mixed", True)])
@pytest.mark.parametrize("shape", FULL, ids=lambda s: "x".join(map(str, s)))
def test_fuller_chips(shape, lens, causal):
    pairs = LENS.get(lens, [(40, 9), (129, 400), (0, 3), (3, 0), (60, 260), (66, 66), (1, 700)])
    q, k, v, cq, ck = make(shape, pairs)
    out = run(q, k, v, cq, ck, causal)
    check(shape, out, q, k, v, cq, ck, causal)
    if lens == "mixed":
        assert not out[:31].any() and not out[cq[3]:cq[4]].any()


@pytest.mark.parametrize("shape", [SHAPES[1], SHAPES[3], SHAPES[5], FULL[1], FULL[5], FULL[9]], ids=str)
def test_strided_rows_and_rows_behind_the_last_prompt(shape):
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    n = 203
    qkv = cu.randn(dtype, 3, n + 9, (H + 2 * G) * D + 32)
    q = qkv[:, :H * D].unflatten(1, (H, D))
    k = qkv[:, H * D:(H + G) * D].unflatten(1, (G, D))
    v = qkv[:, (H + G) * D:(H + 2 * G) * D].unflatten(1, (G, D))
    wide = torch.full((n + 9, H * D + 16), 7.0, dtype=q.dtype, device="cuda")
    out = wide[:, :H * D].unflatten(1, (H, D))
    cq = [0, 120, n]
    run(q, k, v, cq, cq, True, out)
    check(shape, out, q, k, v, cq, cq, True)
    assert (wide[n:] == 7).all() and (wide[:, H * D:] == 7).all()


@pytest.mark.parametrize("shape", [SHAPES[1], FULL[5]], ids=str)
def test_results_beside_the_queries(shape):
    """out in columns of the matrix that holds q, k and v."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    n = 77
    cols = cu.randn(dtype, 4, n, 2 * H + 2 * G, D)
    q, k, v, out = cols[:, :H], cols[:, H:H + G], cols[:, H + G:H + 2 * G], cols[:, H + 2 * G:]
    kept = cols[:, :H + 2 * G].clone()
    run(q, k, v, [0, 40, n], [0, 40, n], True, out)
    check(shape, out, q, k, v, [0, 40, n], [0, 40, n], True)
    assert torch.equal(cols[:, :H + 2 * G], kept)


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1], SHAPES[2], SHAPES[3], SHAPES[6], FULL[0], FULL[3],
                                   FULL[5], FULL[6], FULL[9], FULL[12]], ids=str)
def test_unseen_keys_have_no_influence(shape, where, bad):
    """A key or value that is not finite changes only the rows that see it, bit for bit."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    lens = [(90, 90), (150, 170), (40, 40)]
    q, k, v, cq, ck = make(shape, lens)
    clean = run(q, k, v, cq, ck, True)
    x = {"k": k, "v": v}[where]
    x[ck[1] + 100] = bad           # seen by the rows from 80 of prompt 1 on
    x[ck[2] - 1, :, :3] = bad      # seen by the last row of prompt 1
    x[ck[3] - 1] = bad             # seen by the last row of prompt 2
    out = run(q, k, v, cq, ck, True)
    hidden = torch.ones(cq[-1], dtype=torch.bool, device="cuda")
    hidden[cq[1] + 80:cq[2]] = False
    hidden[-1] = False
    assert torch.equal(out[hidden], clean[hidden])
    if where == "v":
        seen = out[cq[1] + 80:cq[2] - 1]
        assert (seen.isnan() if np.isnan(bad) else seen == bad).all()
        assert (out[-1].isnan() if np.isnan(bad) else out[-1] == bad).all()
    elif np.isnan(bad):
        assert out[cq[1] + 80:cq[2]].isnan().all()


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[2], SHAPES[5], FULL[0], FULL[5], FULL[9]], ids=str)
def test_scores_without_a_softmax_and_rising_ones(shape):
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    n = 300
    q, k, v, cq, ck = make(shape, [(n, n)])
    q[:, :, 0] = 1.0
    # a first run of keys that weigh nothing, then scores that rise by 300 over the prompt
    k[:, :, 0] = torch.linspace(0, 300 * D ** 0.5, n, device="cuda").to(k.dtype)[:, None]
    k[:70, :, 0] = -np.inf
    out = run(q, k, v, cq, ck, True)
    assert out[:70].isnan().all()
    k2 = k.clone()
    k2[:70, :, 0] = 0
    ref = torch.cat([cu.attention(q[i:i + 1], k2[70:i + 1], v[70:i + 1], [i - 69])[0]
                     for i in range(70, n, 23)])
    size = cu.attention(q, k2, v, limits(n, n, True))
    got = out[70:n:23]
    # products up to 300 sqrt(D): scores in fp32 are off by at most S of the definition's bound
    tol = (2.0 ** -7 if dtype == "bf16" else 0) + float((size[2] / size[1].clamp(min=1e-30)).max())
    assert float((got.double() - ref).abs().max()) <= tol * float(v.double().abs().max())


@pytest.mark.parametrize("shape", [SHAPES[0], FULL[0], FULL[1], FULL[2], FULL[3], FULL[5], FULL[10]], ids=str)
def test_jumping_scores_and_large_values(shape):
    """Scores that jump far above what a row has seen, some rows only, now and then; values
    whose sums must not leave the range of fp32 on the way."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    n = 330
    q, k, v, cq, ck = make(shape, [(n, n)])
    q[:, :, 0] = 0
    q[::3, :, 0] = 1.0       # these rows feel the jumps
    k[:, :, 0] = 0
    for i, x in ((40, 12), (41, 300), (100, 305), (170, 900), (260, 890), (300, 5000)):
        k[i, :, 0] = x * D ** 0.5
    v *= 2.0 ** 100
    out = run(q, k, v, cq, ck, True)
    assert out.isfinite().all()
    # products up to 5000 sqrt(D): the scores' own rounding, by the definition's bound
    ref = cu.attention(q, k, v, limits(n, n, True))
    cu.check_attention(out, ref, dtype)
    calm = torch.ones(n, dtype=torch.bool, device="cuda")
    calm[::3] = False
    k[:, :, 0] = 0
    assert torch.equal(run(q, k, v, cq, ck, True)[calm], out[calm])


def test_many_short_prompts():
    """More prompts than one step of the search looks at, some empty."""
    shape = ("bf16", 4, 2, 64)
    lens = [(i * 7 % 4, i * 7 % 4) for i in range(5000)]
    q, k, v, cq, ck = make(shape, lens)
    out = run(q, k, v, cq, ck, True)
    for b in list(range(0, 5000, 311)) + [1, 2, 3, 4997, 4998, 4999]:
        if lens[b][0]:
            sl = slice(cq[b], cq[b + 1])
            ref = cu.attention(q[sl], k[sl], v[sl], limits(*lens[b], True))
            cu.check_attention(out[sl], ref, "bf16")
    assert not (out == 7).all(-1).any()


@pytest.mark.parametrize("shape", [SHAPES[1], FULL[1], FULL[5]], ids=str)
def test_offsets_that_are_wrong_stay_inside(shape):
    """Offsets that start late, fall or leave the tensors touch nothing but the rows of a
    prompt that they do describe; guard rows around every operand keep their values."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    n, pad = 300, 64
    big = [cu.randn(dtype, 5 + i, n + 2 * pad, h, D) for i, h in enumerate((H, G, G))]
    q, k, v = (x[pad:pad + n] for x in big)
    whole = torch.full_like(big[0], 7.0)
    out = whole[pad:pad + n]
    run(q, k, v, [20, 90, 90, 220], [3, 70, 80, 260], True, out)
    assert (whole[:pad + 20] == 7).all() and (whole[pad + 220:] == 7).all()
    for a, b, c, d in ((20, 90, 3, 70), (90, 220, 80, 260)):
        ref = cu.attention(q[a:b], k[c:d], v[c:d], limits(b - a, d - c, True))
        cu.check_attention(out[a:b], ref, dtype)
    for bad in ([0, -5, 700, 20, 1 << 30], [1 << 30, 0, 0, 300, 10], [-9, -1 << 31, 5, 2, 299],
                [300, 200, 100, 50, 0], [150, 10, 290, 10, 2000]):
        run(q, k, v, bad, bad[::-1], True, out)
        run(q, k, v, bad, [0, 100, 200, 250, 300], False, out)
        assert (whole[:pad] == 7).all() and (whole[pad + n:] == 7).all()


@pytest.mark.parametrize("heads,group", [(2, 2), (16, 4)])
def test_rows_far_apart(heads, group):
    """Rows 2^20 elements apart: offsets past 2^32 bytes in every operand."""
    torch = cu.torch_mod()
    D, n, kv = 64, 4400, heads // group
    wide = torch.empty(n, 1 << 20, dtype=torch.bfloat16, device="cuda")
    cols = [0]
    for h in (heads, kv, kv, heads):
        cols.append(cols[-1] + h * D)
    q, k, v, out = (wide[:, a:b].unflatten(1, (-1, D)) for a, b in zip(cols, cols[1:]))
    for i, x in enumerate((q, k, v)):
        x.copy_(cu.randn("bf16", i, *x.shape))
    far = torch.empty(n, 1 << 20, dtype=torch.bfloat16, device="cuda")[:, :heads * D].unflatten(1, (-1, D))
    cq = [0, 100, 4300, n]
    run(q, k, v, cq, cq, True, far)
    dense = run(*(x.contiguous() for x in (q, k, v)), cq, cq, True)
    assert torch.equal(far, dense)
    tail = slice(4300, n)
    cu.check_attention(far[tail], cu.attention(q[tail], k[tail], v[tail], limits(100, 100, True)), "bf16")


def test_scale_and_no_rows():
    torch = cu.torch_mod()
    shape = SHAPES[1]
    q, k, v, cq, ck = make(shape, [(50, 80)])
    check(shape, run(q, k, v, cq, ck, False, scale=0.3), q, k, v, cq, ck, False, 0.3)
    out = run(q, k, v, [0], [0], True)
    assert (out == 7).all()
    out = run(q, k, v, [0, 0, 0], [0, 0, 80], True)
    assert (out == 7).all()


@pytest.mark.parametrize("shape", [SHAPES[0], FULL[1], FULL[6]], ids=str)
def test_replayed_graph_and_other_stream(shape):
    torch = cu.torch_mod()
    from paper_2608_27384_amd.flashvla import prompt_attention
    q, k, v, cq, ck = make(shape, [(150, 150), (111, 190)])
    dq, dk = cu.ints(cq), cu.ints(ck)
    want = run(q, k, v, cq, ck, True)
    out = torch.zeros_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        prompt_attention(q, k, v, dq, dk, out)
    for i in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    q.mul_(0.5)  # the graph reads what the tensors hold when it runs
    want = run(q, k, v, cq, ck, True)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    prompt_attention(q, k, v, dq, dk, out, stream=s)
    s.synchronize()
    assert torch.equal(out, want)


# Prompts of more than 2000 keys on average, one of them longer: (queries, keys)
FAR = [(33, 2700), (900, 2400)]
# (type, heads, kv heads, head dim, causal, the kernel that FAR takes)
FAR_CASES = [("bf16", H, G, D, c, form) for D in (64, 128, 192, 256) for H, G, c, form in (
    (8, 1, True, cu.FEW), (8, 1, False, cu.FEW), (64, 4, True, cu.HALVES), (32, 2, False, cu.HALVES),
    (128, 8, True, cu.TILES), (64, 4, False, cu.TILES))]
FAR_CASES += [("fp32", 128, 8, D, c, cu.FEW) for D in (64, 128, 192, 256) for c in (True, False)]
FAR_CASES += [("fp32", 256, 16, 64, True, cu.TILES), ("fp32", 256, 16, 128, False, cu.TILES),
              ("fp32", 256, 16, 192, True, cu.FEW), ("fp32", 256, 16, 256, False, cu.FEW),
              ("fp32", 288, 18, 192, True, cu.TILES), ("fp32", 288, 18, 256, True, cu.TILES)]


def takes(shape, lens, causal):
    return cu.prompt_form(shape[0], sum(a for a, _ in lens), sum(b for _, b in lens), len(lens),
                          *shape[1:], causal)


def check_some(shape, out, q, k, v, cq, ck, causal, seed=0):
    """Some rows of every prompt, the first and the last ones among them, and some heads."""
    dtype, H, G, D = shape
    rng = np.random.default_rng(seed)
    heads = sorted({0, H // 2, H - 1, *rng.integers(0, H, 2).tolist()})
    kv = [h * G // H for h in heads]
    for b in range(len(cq) - 1):
        nq, nk = int(cq[b + 1] - cq[b]), int(ck[b + 1] - ck[b])
        if nq == 0:
            continue
        rows = sorted({0, 1, 31, 32, 127, 128, nq // 2, nq - 33, nq - 2, nq - 1,
                       *rng.integers(0, nq, 10).tolist()} & set(range(nq)))
        lim = limits(nq, nk, causal)
        at = [int(cq[b]) + r for r in rows]
        ref = cu.attention(q[at][:, heads], k[ck[b]:ck[b + 1]][:, kv], v[ck[b]:ck[b + 1]][:, kv],
                           [lim[r] for r in rows])
        cu.check_attention(out[at][:, heads], ref, dtype)


@pytest.mark.parametrize("case", FAR_CASES, ids=lambda c: "x".join(map(str, c)))
def test_long_prompts(case):
    """Prompts on the far side of the kernels' choice, some rows against the 64-bit form."""
    shape, causal, form = case[:4], case[4], case[5]
    assert takes(shape, FAR, causal) == form
    q, k, v, cq, ck = make(shape, FAR)
    check_some(shape, run(q, k, v, cq, ck, causal), q, k, v, cq, ck, causal)


@pytest.mark.parametrize("case", FAR_CASES, ids=lambda c: "x".join(map(str, c)))
def test_every_key_counts_once(case):
    """With queries of zero every probability is one, and the value of key j in kv head g a one at
    element j + g: a row's result is, times the keys that it sees, how many of them fall on each
    element.  Sums of ones are exact; the quotient's three roundings and the result's own (bf16 2^-8,
    fp32 2^-24) leave less than half a key where an element has at most 43."""
    torch = cu.torch_mod()
    (dtype, H, G, D), causal, form = case[:4], case[4], case[5]
    assert takes(case[:4], FAR, causal) == form
    q, k, v, cq, ck = make(case[:4], FAR)
    q.zero_()
    v.zero_()
    for b in range(2):
        j = torch.arange(FAR[b][1], device="cuda")[:, None]
        g = torch.arange(G, device="cuda")[None]
        v[ck[b]:ck[b + 1]].scatter_(2, ((j + g) % D)[..., None], 1.0)
    out = run(q, k, v, cq, ck, causal)
    d, g = torch.arange(D, device="cuda")[None, None], (torch.arange(H, device="cuda") * G // H)[None, :, None]
    for b, (nq, nk) in enumerate(FAR):
        lim = torch.tensor(limits(nq, nk, causal), device="cuda")[:, None, None]
        want = torch.div(lim - (d - g) % D + D - 1, D, rounding_mode="floor").clamp(min=0)  # keys j = d - g mod D
        assert int(want.max()) <= 43
        got = out[cq[b]:cq[b + 1]].double() * lim
        assert bool(((got - want).abs() <= want * (cu.EPS[dtype] + 2.0 ** -20)).all())


@pytest.mark.parametrize("shape,causal", [(("bf16", 8, 1, 256), False), (("bf16", 8, 1, 256), True),
                                          (("bf16", 16, 4, 128), True), (("fp32", 32, 8, 64), True)], ids=str)
def test_prompts_in_any_order(shape, causal):
    """More row tiles than the chip holds, the longest prompt first, last and anywhere: a prompt's
    result does not depend on its place."""
    torch = cu.torch_mod()
    up = [(300 + 516 * i // 63, 300 + 516 * i // 63) for i in range(64)]
    assert takes(shape, up, causal) == cu.TILES and sum(a for a, _ in up) * shape[1] // 128 > 512
    q, k, v, cq, ck = make(shape, up)
    want = run(q, k, v, cq, ck, causal)
    check_some(shape, want, q, k, v, cq[:3], ck[:3], causal)
    check_some(shape, want[cq[62]:], q[cq[62]:], k[ck[62]:], v[ck[62]:], cq[62:] - cq[62], ck[62:] - ck[62], causal)
    rng = np.random.default_rng(1)
    for order in (np.arange(64)[::-1], rng.permutation(64)):
        at = torch.from_numpy(np.concatenate([np.arange(cq[i], cq[i + 1]) for i in order])).cuda()
        edges = np.cumsum([0] + [up[i][0] for i in order])
        assert torch.equal(run(q[at], k[at], v[at], edges, edges, causal), want[at])


@pytest.mark.parametrize("shape", [("bf16", 128, 16, 64), ("bf16", 128, 16, 128), ("bf16", 128, 16, 192),
                                   ("bf16", 128, 16, 256), ("fp32", 512, 32, 64), ("fp32", 512, 32, 128),
                                   ("fp32", 512, 32, 256)], ids=lambda s: "x".join(map(str, s)))
def test_strided_rows_of_whole_tiles(shape):
    """The kernel of whole tiles on columns of one matrix, its results into columns of another."""
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    n = 300
    cq = np.array([0, 171, n])
    assert takes(shape, [(171, 171), (129, 129)], True) == cu.TILES
    qkv = cu.randn(dtype, 3, n, (H + 2 * G) * D + 32)
    q, k, v = (qkv[:, a * D:b * D].unflatten(1, (-1, D)) for a, b in ((0, H), (H, H + G), (H + G, H + 2 * G)))
    wide = torch.full((n + 5, H * D + 16), 7.0, dtype=q.dtype, device="cuda")
    out = wide[:n, :H * D].unflatten(1, (H, D))
    run(q, k, v, cq, cq, True, out)
    check_some(shape, out, q, k, v, cq, cq, True)
    assert (wide[n:] == 7).all() and (wide[:, H * D:] == 7).all()
    assert torch.equal(out, run(*(x.contiguous() for x in (q, k, v)), cq, cq, True))
