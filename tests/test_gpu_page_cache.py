"""The page cache's upkeep against a plain model of it, step by step, its
refusals (nothing changes), the rotary append against the 64-bit form, and the
whole path as it is used: prompts appended, attended to, continued token by
token, forked, compacted, gathered into the action expert's prefix."""
import random

import numpy as np
import pytest

import context_util as cu

pytestmark = pytest.mark.gpu


def fresh(n_pages, max_seqs, max_pages, page_len=16, layers=2, heads=2, D=64, dtype="bf16", seed=0):
    from paper_2608_27384_amd.flashvla import PageCache
    cache = PageCache.empty(layers, heads, D, n_pages, max_seqs, max_pages, page_len, cu.ttype(dtype))
    cache.k.copy_(cu.randn(dtype, seed, *cache.k.shape))
    cache.v.copy_(cu.randn(dtype, seed + 1, *cache.v.shape))
    return cache, cu.Model(n_pages, max_seqs, max_pages, page_len)


def same(cache, model):
    live = np.arange(model.mp)[None] < -(-model.len // model.pl)[:, None]
    table = cache.table.cpu().numpy()
    assert np.array_equal(cache.length.cpu().numpy(), model.len)
    assert np.array_equal(cache.refs.cpu().numpy(), model.refs)
    assert np.array_equal(table[live], model.table[live])


def state(cache):
    return [x.clone() for x in (cache.table, cache.length, cache.refs, cache.k, cache.v)]


def unchanged(cache, before):
    return all(a.equal(b) for a, b in zip((cache.table, cache.length, cache.refs, cache.k, cache.v),
                                          before))


@pytest.mark.parametrize("n_pages,page_len,dtype,D", [(60, 16, "bf16", 64), (33, 48, "fp32", 64),
                                                      (20000, 16, "bf16", 64), (90, 16, "bf16", 192)])
def test_random_steps(n_pages, page_len, dtype, D):
    """Grown, forked, freed and compacted at random, with lists that fail among them."""
    seqs, width = 24, 12
    cache, model = fresh(n_pages, seqs, width, page_len, dtype=dtype, D=D)
    rng = random.Random(n_pages)
    pools = [cache.k.clone(), cache.v.clone()]
    seen = set()
    for step in range(120):
        op = rng.choice(["grow", "grow", "grow", "fork", "fork", "free", "compact"])
        n = rng.randint(0, 8)
        pick = lambda: [rng.randint(-1 if rng.random() < 0.02 else 0, seqs - 1) for _ in range(n)]
        some = rng.sample(range(seqs), n)
        if op == "grow":
            add = [rng.choice([0, 1, page_len - 1, page_len, 3 * page_len + 1]) for _ in range(n)]
            got, want = cache.grow(cu.ints(some), cu.ints(add)), model.grow(some, add)
        elif op == "fork":
            empty = [s for s in range(seqs) if model.len[s] == 0]
            kids = rng.sample(empty, min(n, len(empty))) if rng.random() < 0.9 else some
            full = [s for s in range(seqs) if model.len[s]] or [0]
            par = [rng.choice(full) for _ in kids] if rng.random() < 0.9 else pick()[:len(kids)]
            kids = kids[:len(par)]
            got = cache.fork(cu.ints(par), cu.ints(kids))
            want, copies = model.fork(par, kids)
            for a, b, r in copies:
                for x in pools:
                    x[:, b, :, :r] = x[:, a, :, :r]
        elif op == "free":
            s = pick()
            got, want = cache.free(cu.ints(s)), model.free(s)
        else:
            got = cache.compact()
            want, moves = model.compact()
            for a, b in moves:
                for x in pools:
                    x[:, b] = x[:, a]
        assert int(got) == want, (step, op)
        seen.add((op, want if op != "compact" else 0))
        same(cache, model)
    assert cache.k.equal(pools[0]) and cache.v.equal(pools[1])
    assert {("grow", 0), ("fork", 0), ("fork", 1), ("free", 0), ("free", 1)} <= seen


def test_refused_lists_change_nothing():
    cache, model = fresh(40, 8, 6)
    assert int(cache.grow(cu.ints([0, 1, 2]), cu.ints([20, 32, 5]))) == 0
    assert int(cache.fork(cu.ints([0]), cu.ints([3]))) == 0
    before = state(cache)
    t = cu.ints
    for call in (lambda: cache.grow(t([0, 0]), t([1, 1])), lambda: cache.grow(t([8]), t([1])),
                 lambda: cache.grow(t([-1]), t([1])), lambda: cache.grow(t([0, 1]), t([1, -1])),
                 lambda: cache.grow(t([0]), t([6 * 16 - 19])), lambda: cache.grow(t([4]), t([2 ** 31 - 1])),
                 lambda: cache.fork(t([0, 1]), t([4, 4])), lambda: cache.fork(t([0]), t([1])),
                 lambda: cache.fork(t([0]), t([0])), lambda: cache.fork(t([4]), t([4])),
                 lambda: cache.fork(t([5, 0]), t([4, 5])), lambda: cache.fork(t([9]), t([4])),
                 lambda: cache.fork(t([0]), t([-7])), lambda: cache.free(t([0, 0])),
                 lambda: cache.free(t([0, 8]))):
        assert int(call()) == 1
        assert unchanged(cache, before)
    # 40 pages, 5 of them held
    assert int(cache.grow(t([4, 5, 6, 7, 0, 1, 2]), t([96, 96, 96, 96, 76, 64, 91]))) == 2
    assert unchanged(cache, before)
    assert int(cache.grow(t([4, 5, 6, 7, 0, 1]), t([96, 96, 96, 96, 76, 64]))) == 0
    assert int(cache.grow(t([2]), t([11 + 3 * 16 + 1]))) == 2
    # a part-filled page that two hold cannot be grown; an entry that is no page cannot be forked
    cache.refs[cache.table[2, 0]] = 2
    before = state(cache)
    assert int(cache.grow(t([2]), t([1]))) == 1 and unchanged(cache, before)
    assert int(cache.grow(t([2]), t([0]))) == 0 and unchanged(cache, before)
    assert int(cache.free(t([7]))) == 0
    cache.table[1, 0] = 40
    before = state(cache)
    assert int(cache.fork(t([1]), t([7]))) == 1 and unchanged(cache, before)
    assert int(cache.free(t([1]))) == 0  # what is no page is skipped


@pytest.mark.parametrize("refs", [0, 2, -1])
def test_a_last_page_that_is_not_the_sequences_alone_is_not_grown_into(refs):
    cache, model = fresh(12, 4, 3)
    assert cache.grow(cu.ints([1]), cu.ints([5])).item() == 0
    cache.refs[0] = refs
    before = state(cache)
    assert cache.grow(cu.ints([1]), cu.ints([1])).item() == 1
    assert unchanged(cache, before)


@pytest.mark.parametrize("n,width", [(1024, 5), (1025, 5), (2600, 4), (40, 300)])
def test_long_lists(n, width):
    """More entries than a plan carries out by itself, and just as many."""
    cache, model = fresh(2 * n * min(width, 5) + 30000, 2 * n + 3, width, layers=1, heads=1)
    rng = random.Random(n)
    seqs = rng.sample(range(n), n)
    for most in (40, 20):
        add = [rng.choice([0, 1, 16, 17, rng.randint(0, most)]) for _ in seqs]
        if width > 100 and most == 40:
            add[3], add[30] = 4000, 2500
        assert int(cache.grow(cu.ints(seqs), cu.ints(add))) == model.grow(seqs, add) == 0
        same(cache, model)
    par, kids = rng.choices(range(n), k=n), rng.sample(range(n, 2 * n + 3), n)
    assert int(cache.fork(cu.ints(par), cu.ints(kids))) == 0
    assert model.fork(par, kids)[0] == 0
    same(cache, model)
    assert int(cache.free(cu.ints(seqs + seqs[:1]))) == 1
    same(cache, model)
    assert int(cache.free(cu.ints(seqs[::-1]))) == model.free(seqs) == 0
    same(cache, model)
    assert (cache.table[:n] == -1).all()
    assert int(cache.compact()) == model.compact()[0]
    same(cache, model)


def test_empty_lists():
    torch = cu.torch_mod()
    cache, model = fresh(10, 4, 4)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    before = state(cache)
    st = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    for call in (lambda: cache.grow(none, none, st), lambda: cache.fork(none, none, st),
                 lambda: cache.free(none, st)):
        st.fill_(9)
        call()
        assert int(st) == 0
    assert int(cache.compact()) == 0
    out = torch.empty(2, 0, 5, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache.gather(none, out, out)
    assert unchanged(cache, before)


@pytest.mark.parametrize("page_len,dtype,D", [(16, "bf16", 256), (48, "fp32", 64), (128, "bf16", 192)])
def test_gather(page_len, dtype, D):
    torch = cu.torch_mod()
    cache, model = fresh(80, 6, 9, page_len, layers=3, heads=2, D=D, dtype=dtype)
    lens = [1, page_len, 3 * page_len + 5, 0, 7 * page_len - 1]
    cache.grow(cu.ints(range(5)), cu.ints(lens))
    cache.free(cu.ints([1]))
    cache.grow(cu.ints([1, 5]), cu.ints([page_len + 1, 2]))
    lens = [1, page_len + 1, 3 * page_len + 5, 0, 7 * page_len - 1, 2]
    seqs, ld = [4, 0, 2, -1, 2, 3, 6, 1], 5 * page_len + 3
    k = cu.randn(dtype, 7, 3, len(seqs), ld, 2, D)
    v = cu.randn(dtype, 8, 3, len(seqs), ld, 2, D)
    want = [k.clone(), v.clone()]
    cache.table[2, 1] = -1  # a hole
    for i, s in enumerate(seqs):
        for r in range(min(lens[s], ld) if 0 <= s < 6 else 0):
            p = int(cache.table[s, r // page_len])
            if p >= 0:
                want[0][:, i, r] = cache.k[:, p, :, r % page_len]
                want[1][:, i, r] = cache.v[:, p, :, r % page_len]
    cache.gather(cu.ints(seqs), k, v)
    assert k.equal(want[0]) and v.equal(want[1])


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("fp32", 192)])
def test_copies_of_more_than_the_caches_hold(dtype, D):
    """Gathered and compacted in a pool of more than half a gigabyte."""
    torch = cu.torch_mod()
    G, L = 2, 2
    token = 2 * L * G * D * (2 if dtype == "bf16" else 4)
    pages = (1 << 29) // (16 * token) + 9
    cache, model = fresh(pages, 5, pages, layers=L, heads=G, D=D, dtype=dtype)
    lens = [70, (pages // 2) * 16 - 3, 1, 0, pages * 5 + 1]
    assert int(cache.grow(cu.ints(range(5)), cu.ints(lens))) == 0
    model.grow(list(range(5)), lens)

    def gathered(seqs, ld):
        k, v = (torch.full((L, len(seqs), ld, G, D), 7.0, dtype=cache.k.dtype, device="cuda")
                for _ in range(2))
        cache.gather(cu.ints(seqs), k, v)
        return k, v

    ld = lens[1] + 40
    got = gathered([4, 1], ld)
    table = cache.table.long()
    for out, pool in zip(got, (cache.k, cache.v)):
        for i, s in enumerate((4, 1)):
            want = pool[:, table[s, :-(-lens[s] // 16)]].transpose(2, 3).reshape(L, -1, G, D)
            assert out[:, i, :lens[s]].equal(want[:, :lens[s]]) and bool((out[:, i, lens[s]:] == 7).all())
    assert int(cache.free(cu.ints([1]))) == 0
    model.free([1])
    before = gathered([4, 0, 2], ld)
    used, _ = model.compact()
    assert int(cache.compact()) == used
    same(cache, model)
    after = gathered([4, 0, 2], ld)
    assert before[0].equal(after[0]) and before[1].equal(after[1])


def test_captured_upkeep():
    """Free, fork, grow and compact in one graph, replayed on bookkeeping that changes."""
    torch = cu.torch_mod()
    cache, model = fresh(64, 8, 8, seed=5)
    a, b, c = cu.ints([1]), cu.ints([0, 0]), cu.ints([5, 6])
    add = cu.ints([3, 20])
    cache.grow(cu.ints([0, 1, 2]), cu.ints([40, 33, 17]))
    model.grow([0, 1, 2], [40, 33, 17])
    g = torch.cuda.CUDAGraph()
    before = state(cache)
    with torch.cuda.graph(g):
        st = [cache.free(a), cache.fork(b, c), cache.grow(c, add), cache.compact()]
    assert unchanged(cache, before)
    pools = [cache.k.clone(), cache.v.clone()]
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
        want = [model.free([1])]
        s, copies = model.fork([0, 0], [5, 6])
        want += [s, model.grow([5, 6], [3, 20])]
        u, moves = model.compact()
        assert [int(x) for x in st] == want + [u]
        for x in pools:
            for p, q, r in copies:
                x[:, q, :, :r] = x[:, p, :, :r]
            for p, q in moves:
                x[:, q] = x[:, p]
        same(cache, model)
        assert cache.k.equal(pools[0]) and cache.v.equal(pools[1])
        cache.free(cu.ints([5, 6]))
        model.free([5, 6])
        cache.grow(cu.ints([1]), cu.ints([20]))
        model.grow([1], [20])


ROPE = [("bf16", 8, 1, 256, (32, 48, 48)), ("bf16", 4, 2, 64, (5, 13, 14)), ("fp32", 3, 1, 192, (96,)),
        ("bf16", 8, 8, 128, (1, 0, 60, 3)), ("fp32", 4, 2, 128, (30, 34)), ("bf16", 6, 2, 192, (96, 0))]


@pytest.mark.parametrize("n", [1, 7, 2053, 8197])
@pytest.mark.parametrize("shape", ROPE, ids=lambda s: "x".join(map(str, s)))
def test_rotary_append(shape, n):
    torch = cu.torch_mod()
    dtype, H, G, D, sections = shape
    rng = np.random.default_rng(n)
    lens = [n // 3, n - n // 3]
    cache, model = fresh(n // 16 + 8, 3, n // 16 + 3, 16, heads=G, D=D, dtype=dtype)
    cache.grow(cu.ints([0, 2]), cu.ints(lens))
    seqs = np.repeat([0, 2], lens)
    at = np.concatenate([np.arange(x) for x in lens])
    order = rng.permutation(n)
    seqs, at = seqs[order], at[order]
    skip = np.zeros(n, bool)
    if n > 7:  # padding, places that do not exist
        seqs[3], seqs[9], at[11], at[20] = -1, 3, -1, 1 << 30
        skip[[3, 9, 11, 20]] = True
    pos = rng.integers(-50, 4000, (len(sections), n))
    pos[0, 0], pos[-1, n // 2] = 1 << 24, -(1 << 20)
    qkv = cu.randn(dtype, n, n, H + 2 * G, D)
    q, k, v = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
    qo = torch.zeros(n, H, D, dtype=q.dtype, device="cuda")
    ko = torch.zeros(n, G, D, dtype=q.dtype, device="cuda")
    want = [cache.k.clone(), cache.v.clone()]
    cache.append(1, q, k, v, cu.ints(pos), cu.ints(seqs), cu.ints(at), sections, 5e5, qo, ko)
    # an angle of x is off by x 2^-50 at most: 64-bit powers, products and fractions
    far = float(np.abs(pos).max()) * 2.0 ** -50
    cu.check_rotated(qo, cu.rotate(q, pos, sections, 5e5), dtype, far)
    cu.check_rotated(ko, cu.rotate(k, pos, sections, 5e5), dtype, far)
    keep = torch.from_numpy(np.nonzero(~skip)[0]).cuda()
    s, p = (torch.from_numpy(x[~skip]).cuda() for x in (seqs, at))
    page = cache.table[s, p // 16].long()
    want[0][1, page, :, p % 16] = ko[keep]
    want[1][1, page, :, p % 16] = v[keep]
    assert cache.k.equal(want[0]) and cache.v.equal(want[1])
    # in place, and without a cache
    from paper_2608_27384_amd.flashvla import rope
    q2, k2 = (torch.zeros_like(x).contiguous() for x in (qo, ko))
    rope(q, k, cu.ints(pos), sections, q2, k2, 5e5)
    assert q2.equal(qo) and k2.equal(ko)
    clean = v.clone()
    cache.append(0, q, k, v, cu.ints(pos), cu.ints(seqs), cu.ints(at), sections, 5e5, None, k)
    assert q.equal(qo) and k.equal(ko) and v.equal(clean)
    assert cache.k[0, page, :, p % 16].equal(ko[keep])


def test_rotary_rows_far_apart():
    """Rows 2^20 elements apart: offsets past 2^32 bytes."""
    torch = cu.torch_mod()
    from paper_2608_27384_amd.flashvla import rope
    n, D = 4300, 64
    wide = torch.empty(n, 1 << 20, dtype=torch.bfloat16, device="cuda")
    q, k = wide[:, :2 * D].unflatten(1, (2, D)), wide[:, 2 * D:3 * D].unflatten(1, (1, D))
    q.copy_(cu.randn("bf16", 1, n, 2, D))
    k.copy_(cu.randn("bf16", 2, n, 1, D))
    pos = cu.ints([np.arange(n)])
    qo, ko = torch.empty(n, 2, D, dtype=q.dtype, device="cuda"), torch.empty(n, 1, D, dtype=q.dtype, device="cuda")
    rope(q, k, pos, (D // 2,), qo, ko)
    ref = cu.rotate(q.contiguous(), [np.arange(n)], (D // 2,), 1e4)
    cu.check_rotated(qo, ref, "bf16", n * 2.0 ** -50)
    rope(q, k, pos, (D // 2,), q, k)
    assert q.equal(qo) and k.equal(ko)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rotary_into_columns_of_one_matrix(dtype):
    """Queries and keys rotated into their columns of one packed matrix, the other columns left."""
    torch = cu.torch_mod()
    from paper_2608_27384_amd.flashvla import rope
    n, H, G, D = 37, 4, 2, 64
    qkv = cu.randn(dtype, 5, n, (H + 2 * G) * D)
    q, k = qkv[:, :H * D].unflatten(1, (H, D)), qkv[:, H * D:(H + G) * D].unflatten(1, (G, D))
    pos = cu.ints([np.arange(n)])
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    rope(q, k, pos, (D // 2,), qo, ko)
    for order in ((0, H), (G, 0)):  # queries first, keys first
        packed = torch.full((n, (H + 2 * G) * D), 7.0, dtype=qkv.dtype, device="cuda")
        heads = packed.unflatten(1, (H + 2 * G, D))
        rope(q, k, pos, (D // 2,), heads[:, order[0]:order[0] + H], heads[:, order[1]:order[1] + G])
        assert heads[:, order[0]:order[0] + H].equal(qo) and heads[:, order[1]:order[1] + G].equal(ko)
        assert (heads[:, H + G:] == 7).all()


def test_one_axis_is_the_action_tokens_rotation():
    """Equal positions on every axis turn as one axis does."""
    torch = cu.torch_mod()
    from paper_2608_27384_amd.flashvla import rope
    q, k = cu.randn("bf16", 0, 100, 8, 256), cu.randn("bf16", 1, 100, 1, 256)
    a, b = torch.empty_like(q), torch.empty_like(q)
    p = np.arange(100)
    rope(q, k, cu.ints([p, p, p]), (20, 50, 58), a)
    rope(q, k, cu.ints([p]), (128,), b)
    assert a.equal(b)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_context_of_a_run(dtype):
    """Three observations, two layers: append, attend, two more tokens each over the pages,
    one sequence forked, one freed, the pool compacted; the gathered context is what the
    action expert then decodes against."""
    import oracle
    import synth
    from gpu_util import Case, host, rel_err, tol
    from paper_2608_27384_amd.flashvla import PageCache, prompt_attention
    torch = cu.torch_mod()
    w = synth.workload("small_bf16_b3").replace(prefix_len=140, dtype=dtype)
    H, G, D, L = w.n_q_heads, w.n_kv_heads, w.head_dim, w.n_layers
    lens, sections = [90, 33, 128], (16, 24, 24)
    cache = PageCache.empty(L, G, D, 64, 6, 10, 16, cu.ttype(dtype))
    cache.k.fill_(float("nan"))
    cache.v.fill_(float("nan"))
    seqs = [0, 1, 2]
    keys, values = [[[], [], []] for _ in range(L)], [[[], [], []] for _ in range(L)]

    def step(lens_new, starts, seed):
        n = sum(lens_new)
        assert int(cache.grow(cu.ints(seqs), cu.ints(lens_new))) == 0
        sq = np.repeat(seqs, lens_new)
        at = np.concatenate([s + np.arange(x) for s, x in zip(starts, lens_new)])
        pos = np.stack([at, at // 4, at % 4])
        edges = np.cumsum([0] + lens_new)
        outs = []
        for l in range(L):
            q, k, v = (cu.randn(dtype, seed + 3 * l + i, n, x, D) for i, x in enumerate((H, G, G)))
            ko = torch.empty_like(k)
            cache.append(l, q, k, v, cu.ints(pos), cu.ints(sq), cu.ints(at), sections, k_out=ko)
            for b in range(3):
                keys[l][b].append(ko[edges[b]:edges[b + 1]])
                values[l][b].append(v[edges[b]:edges[b + 1]])
            out = torch.empty_like(q)
            if n > 3:
                prompt_attention(q, ko, v, cu.ints(edges), cu.ints(edges), out)
            else:
                cache.attend(l, q, cu.ints(seqs), out)
            outs.append((q, out, edges))
        return outs

    for outs, starts in ((step(lens, [0, 0, 0], 100), [0, 0, 0]),
                         (step([1, 1, 1], lens, 200), lens),
                         (step([1, 1, 1], [x + 1 for x in lens], 300), [x + 1 for x in lens])):
        for l, (q, out, edges) in enumerate(outs):
            for b in range(3):
                n = edges[b + 1] - edges[b]
                kk, vv = torch.cat(keys[l][b])[:starts[b] + n], torch.cat(values[l][b])[:starts[b] + n]
                ref = cu.attention(q[edges[b]:edges[b + 1]], kk, vv, [starts[b] + i + 1 for i in range(n)])
                cu.check_attention(out[edges[b]:edges[b + 1]], ref, dtype)
    assert int(cache.fork(cu.ints([0]), cu.ints([4]))) == 0
    assert int(cache.free(cu.ints([0]))) == 0
    cache.compact()
    case = Case(w, lens=[35, 92, 130])
    try:
        shape = (L, 3, 140, G, D)
        kd, vd = (torch.full(shape, float("nan"), dtype=cu.ttype(dtype), device="cuda") for _ in range(2))
        cache.gather(cu.ints([1, 4, 2]), kd, vd)
        for i, b in enumerate((1, 0, 2)):
            for l in range(L):
                assert kd[l, i, :lens[b] + 2].equal(torch.cat(keys[l][b]))
                assert vd[l, i, :lens[b] + 2].equal(torch.cat(values[l][b]))
        case.ex.set_prefix(kd, vd, case.lens)
        case.k, case.v = (np.nan_to_num(x.float().cpu().numpy()) for x in (kd, vd))
        new, ref = oracle.decode_step(case.x, case.t, case.k, case.v, case.lens, case.W, w,
                                      noise_seed=0, step=0)
        case.ex.decode_step(case.xd, case.td, case.out)
        got = host(case.out)
        for b in range(3):
            assert rel_err(got[b], ref[b]) < tol(w)
    finally:
        case.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_captured_token_step(dtype):
    """A token step of two layers (room, rotary append where the lengths say, attention) in one
    graph, replayed over page ends with the eager steps of another cache between."""
    torch = cu.torch_mod()
    H, G, D, L, n = 4, 2, 64, 2, 5
    sections = (D // 2,)
    runs = []
    for _ in range(2):
        cache, _ = fresh(60, 6, 8, 16, layers=L, heads=G, D=D, dtype=dtype, seed=3)
        cache.grow(cu.ints(range(6)), cu.ints([1, 15, 16, 0, 31, 40]))
        runs.append(cache)
    seqs = cu.ints([4, 0, 2, 1, -1])
    live = seqs.long()[:4]
    x = [cu.randn(dtype, 20 + i, n, h, D) for i, h in enumerate((H, G, G))]

    def buffers():
        return dict(q=torch.empty_like(x[0]), out=[torch.zeros_like(x[0]) for _ in range(L)],
                    at=torch.zeros(n, dtype=torch.int32, device="cuda"),
                    one=torch.ones(4, dtype=torch.int32, device="cuda"), few=seqs[:4].clone(),
                    status=torch.empty(1, dtype=torch.int32, device="cuda"))

    def step(cache, b):
        cache.grow(b["few"], b["one"], b["status"])
        b["at"][:4].copy_(cache.length.index_select(0, live) - 1)
        for l in range(L):
            cache.append(l, x[0], x[1], x[2], b["at"].view(1, n), seqs, b["at"], sections, q_out=b["q"])
            cache.attend(l, b["q"], seqs, b["out"][l])

    a, b = buffers(), buffers()
    before = state(runs[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(runs[0], a)
    assert unchanged(runs[0], before)
    for i in range(20):
        for t, scale in zip(x, (0.9, 1.1, -0.8)):
            t.mul_(scale)
        g.replay()
        step(runs[1], b)
        torch.cuda.synchronize()
        assert a["status"].item() == 0 and b["status"].item() == 0
        assert unchanged(runs[0], state(runs[1]))
        for l in range(L):
            assert a["out"][l].equal(b["out"][l]) and (a["out"][l][4] == 0).all()
    assert runs[0].length.tolist() == [21, 35, 36, 0, 51, 40]


@pytest.mark.parametrize("poison", [0, 1, 7, 15, 39, -1, 1 << 30])
@pytest.mark.parametrize("refs", [0, -1])
def test_compaction_leaves_entries_on_pages_that_nobody_holds(refs, poison):
    """A live entry whose page has no holder, past the pages in use, keeps its number whatever an
    earlier call left in the workspace; the others move."""
    import ctypes
    from paper_2608_27384_amd import flashvla as fvb
    torch = cu.torch_mod()
    cache, model = fresh(40, 4, 12)
    for s, n in ((0, 160), (1, 80), (2, 76)):
        assert cache.grow(cu.ints([s]), cu.ints([n])).item() == model.grow([s], [n]) == 0
    assert cache.free(cu.ints([0])).item() == model.free([0]) == 0
    lost = int(model.table[1, 2])
    cache.refs[lost] = refs
    model.refs[lost] = 0
    want = model.compact()[0]
    model.refs[lost] = refs
    work = torch.full((cache.work_bytes // 4,), poison, dtype=torch.int32, device="cuda")
    used = torch.empty(1, dtype=torch.int32, device="cuda")
    st = fvb.lib().fv_pages_compact(ctypes.byref(cache.c), used.data_ptr(), work.data_ptr(),
                                    torch.cuda.current_stream().cuda_stream)
    assert st == 0 and used.item() == want == 9
    assert cache.table[1, 2].item() == lost == 12
    same(cache, model)


def test_written_tensors_move_their_versions():
    """A tensor that autograd keeps for a backward pass and a call then overwrites is noticed."""
    torch = cu.torch_mod()
    from paper_2608_27384_amd.flashvla import prompt_attention, rope
    cache, _ = fresh(20, 4, 4)
    q, k, v = (cu.randn("bf16", i, 5, h, 64) for i, h in enumerate((4, 2, 2)))
    out, ko = torch.empty_like(q), torch.empty_like(k)
    at, seqs, cum = cu.ints(range(5)), cu.ints([0] * 5), cu.ints([0, 5])
    kd, vd = (torch.empty(2, 1, 5, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    st = torch.empty(1, dtype=torch.int32, device="cuda")
    books, pools = [cache.table, cache.length, cache.refs, st], [cache.k, cache.v]
    every = books + pools + [q, k, v, out, ko, kd, vd, at, seqs, cum]

    def moved(call):
        before = [t._version for t in every]
        call()
        return [t for t, b in zip(every, before) if t._version != b]

    def same(got, want):
        assert [t.data_ptr() for t in got] == [t.data_ptr() for t in every if any(t is w for w in want)]

    same(moved(lambda: cache.grow(cu.ints([0]), cu.ints([5]), st)), books)
    same(moved(lambda: cache.append(0, q, k, v, at[None], seqs, at, (32,))), pools + [q])
    same(moved(lambda: cache.append(1, q, k, v, at[None], seqs, at, (32,), q_out=out, k_out=ko)), pools + [out, ko])
    same(moved(lambda: rope(q, k, at[None], (32,), out)), [out])
    same(moved(lambda: prompt_attention(q, k, v, cum, cum, out)), [out])
    same(moved(lambda: cache.attend(0, q, seqs, out)), [out])
    same(moved(lambda: cache.fork(cu.ints([0]), cu.ints([1]), st)), books + pools)
    same(moved(lambda: cache.gather(cu.ints([0]), kd, vd)), [kd, vd])
    same(moved(lambda: cache.compact(st)), books + pools)
    same(moved(lambda: cache.free(cu.ints([0]), st)), books)
    w = torch.ones(4, 64, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    y = (q * w).sum()  # keeps q
    cache.append(0, q, k, v, at[None], seqs, at, (32,))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    with torch.inference_mode():  # tensors without versions
        z = torch.empty_like(q)
        prompt_attention(q, k, v, cum, cum, z)
        assert z.isfinite().all()


@pytest.mark.parametrize("dtype,D,theta", [("bf16", 256, 1e4), ("fp32", 64, 1e4), ("fp32", 128, 5e5)])
def test_one_axis_against_the_action_experts_rotation(dtype, D, theta):
    """The oracle's rotation of the action tokens in 64 bits, at positions of their arena."""
    import oracle.flashvla as oracle
    torch = cu.torch_mod()
    from paper_2608_27384_amd.flashvla import rope
    n = 301
    q, k = cu.randn(dtype, 0, n, 3, D), cu.randn(dtype, 1, n, 1, D)
    p = np.concatenate([np.arange(200), 28672 + np.arange(101)])
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    rope(q, k, cu.ints([p]), (D // 2,), qo, ko, theta)
    for x, got in ((q, qo), (k, ko)):
        want = torch.from_numpy(oracle.rope_tokens(x.double().cpu().numpy(), p, theta)).cuda()
        _, size, whole = cu.rotate(x, [p], (D // 2,), theta)
        cu.check_rotated(got, (want, size, whole), dtype, float(p.max()) * 2.0 ** -50)
