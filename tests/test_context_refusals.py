"""What the observation context's operators refuse: at the C boundary from the
arguments alone (no GPU is touched), and in the binding from the tensors'
shapes, types and strides."""
import ctypes

import pytest

from paper_2608_27384_amd import flashvla as fvb

P = 1 << 20  # an aligned address that is never read


def cache(**kw):
    c = fvb.FvPages(fvb.FV_BF16, 2, 2, 64, 16, 10, 4, 3, P, P, P, P, P)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rope_args(**kw):
    a = fvb.FvRopeArgs(P, P << 1, P << 2, P << 3, P << 4, 256, 128, 128, 256, 128, P, P, P, 5, 4, 2, 64,
                       fvb.FV_BF16, 0, 3, (ctypes.c_int32 * 4)(8, 12, 12), 1e4)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def prompt_args(**kw):
    a = fvb.FvPromptArgs(P, P << 1, P << 2, P << 3, 256, 128, 128, 256, P, P, 2, 9, 9, 4, 2, 64,
                         fvb.FV_BF16, 1, 0.125)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def paged_args(**kw):
    a = fvb.FvPagedArgs(P, P << 1, 256, 256, P, 3, 4, 0, 0, 0.125, None, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def refused(st, word=""):
    assert st == fvb.FV_ERR_INVALID_ARG
    msg = fvb.lib().fv_context_error().decode()
    assert msg and word in msg, msg


def test_structures_match_the_header():
    assert ctypes.sizeof(fvb.FvPages) == 32 + 5 * 8
    assert ctypes.sizeof(fvb.FvRopeArgs) == 5 * 8 + 24 + 3 * 8 + 12 * 4
    assert ctypes.sizeof(fvb.FvPromptArgs) == 4 * 8 + 16 + 16 + 9 * 4 + 4
    assert ctypes.sizeof(fvb.FvPagedArgs) == 16 + 8 + 8 + 16 + 8 + 8 + 8


CACHES = [("dtype", 2), ("dtype", -1), ("n_layers", 0), ("n_layers", 1025), ("n_kv_heads", 0),
          ("head_dim", 80), ("page_len", 8), ("page_len", 24), ("page_len", 272), ("page_len", 0),
          ("n_pages", 0), ("n_pages", (1 << 20) + 1), ("max_seqs", 0), ("max_seqs", 65537),
          ("max_pages", 0), ("max_pages", 65537), ("k", None), ("v", P + 8), ("table", None),
          ("len", P + 2), ("refs", None)]


@pytest.mark.parametrize("field,value", CACHES)
def test_caches(field, value):
    L, c = fvb.lib(), cache(**{field: value})
    b, n = ctypes.byref(c), ctypes.c_size_t()
    refused(L.fv_pages_workspace(b, ctypes.byref(n)))
    refused(L.fv_pages_grow(b, P, P, 1, P, P, None))
    refused(L.fv_pages_fork(b, P, P, 1, P, P, None))
    refused(L.fv_pages_free(b, P, 1, P, None))
    refused(L.fv_pages_compact(b, P, P, None))
    refused(L.fv_pages_gather(b, P, 1, 5, P, P, None))
    refused(L.fv_paged_attention(ctypes.byref(paged_args()), b, None))
    refused(L.fv_rope_append(ctypes.byref(rope_args()), b, None))


@pytest.mark.parametrize("kw", [
    dict(dtype=3), dict(head_dim=32), dict(n_q_heads=3), dict(n_q_heads=0), dict(n_q_heads=1026),
    dict(n=-1), dict(n_axes=0), dict(n_axes=5), dict(sections=(ctypes.c_int32 * 4)(8, 12, 11)),
    dict(sections=(ctypes.c_int32 * 4)(-8, 28, 12)), dict(theta=0.0), dict(theta=float("nan")),
    dict(theta=float("inf")), dict(layer=2), dict(layer=-1), dict(n_kv_heads=1, ldk=64), dict(q=None),
    dict(k=P + 4), dict(v=None), dict(q_out=None), dict(ldq=255), dict(ldq=248), dict(ldk=120),
    dict(ldv=(1 << 20) + 8), dict(ldq_out=252), dict(ldk_out=64), dict(pos=None), dict(seqs=None),
    dict(at=P + 1), dict(q_out=P + 64), dict(q_out=P << 1), dict(k_out=P << 2), dict(k_out=P << 3),
    dict(q_out=P, ldq_out=264), dict(dtype=fvb.FV_FP32)], ids=str)
def test_rope(kw):
    refused(fvb.lib().fv_rope_append(ctypes.byref(rope_args(**kw)), ctypes.byref(cache()), None))


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(head_dim=512), dict(n_q_heads=5), dict(n_kv_heads=0), dict(n_seqs=-1),
    dict(n_seqs=65537), dict(n_q=-1), dict(n_k=-1), dict(causal=2), dict(scale=0.0), dict(scale=-1.0),
    dict(scale=float("inf")), dict(scale=float("nan")), dict(q=None), dict(k=None), dict(v=P + 2),
    dict(out=None), dict(ldq=128), dict(ldk=130), dict(ldo=(1 << 20) + 8), dict(cu_q=None),
    dict(cu_k=P + 3), dict(out=P), dict(out=(P << 1) + 1024), dict(out=P << 2),
    dict(n_q=1 << 30)], ids=str)
def test_prompts(kw):
    refused(fvb.lib().fv_prompt_attention(ctypes.byref(prompt_args(**kw)), None))


@pytest.mark.parametrize("kw", [
    dict(n=-1), dict(n=65537), dict(n_q_heads=3), dict(max_len=-1), dict(layer=2), dict(scale=0.0),
    dict(q=None), dict(out=P + 8), dict(out=P + 512), dict(ldq=128), dict(ldo=260), dict(seqs=None)],
    ids=str)
def test_paged(kw):
    refused(fvb.lib().fv_paged_attention(ctypes.byref(paged_args(**kw)), ctypes.byref(cache()), None))


def test_paged_workspace_too_small():
    L, c = fvb.lib(), cache(max_pages=4000)
    n = ctypes.c_size_t()
    a = paged_args()
    assert L.fv_paged_attention_workspace(ctypes.byref(a), ctypes.byref(c), ctypes.byref(n)) == 0
    assert n.value > 0
    refused(L.fv_paged_attention(ctypes.byref(a), ctypes.byref(c), None), "work")
    a = paged_args(work=P << 4, work_bytes=n.value - 1)
    refused(L.fv_paged_attention(ctypes.byref(a), ctypes.byref(c), None), "work")


def test_lists():
    L, c = fvb.lib(), cache()
    b = ctypes.byref(c)
    for n in (-1, 5):
        refused(L.fv_pages_grow(b, P, P, n, P, P, None))
        refused(L.fv_pages_fork(b, P, P, n, P, P, None))
        refused(L.fv_pages_free(b, P, n, P, None))
    refused(L.fv_pages_grow(b, P, None, 1, P, P, None))
    refused(L.fv_pages_grow(b, P, P, 1, None, P, None))
    refused(L.fv_pages_grow(b, P, P, 1, P, P + 4, None))
    refused(L.fv_pages_fork(b, None, P, 1, P, P, None))
    refused(L.fv_pages_free(b, P + 1, 1, P, None))
    refused(L.fv_pages_compact(b, None, P, None))
    refused(L.fv_pages_compact(b, P, None, None))
    refused(L.fv_pages_gather(b, P, -1, 5, P, P, None))
    refused(L.fv_pages_gather(b, P, 1, -5, P, P, None))
    refused(L.fv_pages_gather(b, P, 1, 5, P + 8, P, None))


def test_null_arguments_and_the_message():
    L = fvb.lib()
    assert L.fv_rope_append(None, None, None) == fvb.FV_ERR_INVALID_ARG
    assert L.fv_prompt_attention(None, None) == fvb.FV_ERR_INVALID_ARG
    assert L.fv_paged_attention(None, None, None) == fvb.FV_ERR_INVALID_ARG
    assert L.fv_pages_workspace(None, None) == fvb.FV_ERR_INVALID_ARG
    assert b"NULL" in L.fv_context_error()
    # calls of nothing touch no GPU and succeed
    assert L.fv_prompt_attention(ctypes.byref(prompt_args(n_q=0, q=None)), None) == 0
    assert L.fv_paged_attention(ctypes.byref(paged_args(n=0)), ctypes.byref(cache()), None) == 0
    assert L.fv_rope_append(ctypes.byref(rope_args(n=0)), None, None) == 0
    assert L.fv_context_error() == b""


def test_binding_refuses_tensors():
    torch = pytest.importorskip("torch")
    q, k = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64)
    cu = torch.tensor([0, 3], dtype=torch.int32)

    def no(fn, *a, **kw):
        with pytest.raises(fvb.FlashVLAError) as e:
            fn(*a, **kw)
        assert e.value.status == fvb.FV_ERR_INVALID_ARG

    pa = fvb.prompt_attention
    no(pa, q, k, k.clone(), cu, cu, torch.zeros_like(q))  # not on a GPU
    no(pa, q.half(), k, k, cu, cu, q)
    no(pa, q, k.bfloat16(), k, cu, cu, q)
    no(pa, q, k, k[:2], cu, cu, q)
    no(pa, q, k, k, cu, cu, q[:, :2])
    no(pa, q.transpose(0, 1), k, k, cu, cu, q)
    no(pa, q, k[..., :32], k[..., :32], cu, cu, q)
    pool, refs = torch.zeros(2, 10, 2, 16, 64), torch.zeros(10, dtype=torch.int32)
    table, length = torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    c = fvb.PageCache(pool, pool.clone(), table, length, refs)
    no(fvb.PageCache, pool, pool[:1], table, length, refs)
    no(fvb.PageCache, pool.half(), pool.half(), table, length, refs)
    no(fvb.PageCache, pool, pool.clone(), table.long(), length, refs)
    no(fvb.PageCache, pool, pool.clone(), table, length[:3], refs)
    no(fvb.PageCache, pool, pool.clone(), table, length, refs[:9])
    seqs = torch.zeros(3, dtype=torch.int32)
    no(c.attend, 0, q, seqs, q.clone())
    no(c.attend, 0, q.bfloat16(), seqs, q.bfloat16())
    no(c.attend, 0, q, seqs.long(), q.clone())
    no(c.attend, 0, q, seqs[:2], q.clone())
    no(c.grow, seqs, seqs[:2])
    no(c.grow, seqs, seqs)
    no(c.gather, seqs, torch.zeros(2, 3, 5, 2, 64), torch.zeros(2, 3, 6, 2, 64))
    no(c.gather, seqs, torch.zeros(1, 3, 5, 2, 64), torch.zeros(1, 3, 5, 2, 64))
    pos = torch.zeros(3, 3, dtype=torch.int32)
    no(c.append, 0, q, k, None, pos, seqs, seqs, (8, 12, 12))
    no(c.append, 0, q, k, k, pos[:2], seqs, seqs, (8, 12, 12))
    no(c.append, 0, q, k, k, pos, seqs, seqs, (8, 8, 4, 4, 8))
    no(fvb.rope, q, k[:2], pos, (8, 12, 12), q)


def test_sizes_beyond_a_launch():
    """Sizes whose grid would hold 2^32 threads or more are refused before anything is launched."""
    L, ref = fvb.lib(), ctypes.byref
    refused(L.fv_rope_append(ref(rope_args(n=(1 << 26) + 1)), None, None), "2^26")
    refused(L.fv_prompt_attention(ref(prompt_args(n_q=(1 << 28) + 1)), None), "2^30")
    wide = dict(n_seqs=65536, n_q_heads=128, n_kv_heads=128, ldq=8192, ldk=8192, ldv=8192, ldo=8192)
    refused(L.fv_prompt_attention(ref(prompt_args(**wide)), None), "2^22")
    many = cache(n_kv_heads=128, max_seqs=65536, max_pages=65536)
    n = ctypes.c_size_t()
    refused(L.fv_paged_attention_workspace(ref(paged_args(n=65536, n_q_heads=128)), ref(many), ref(n)),
            "2^22")
    refused(L.fv_paged_attention(ref(paged_args(n=65536, n_q_heads=128)), ref(many), None), "2^22")
    # the most rows that are taken: two chunks each, 2^23 workgroups
    assert L.fv_paged_attention_workspace(ref(paged_args(n=32768, n_q_heads=128)), ref(many), ref(n)) == 0
    assert n.value == 2 * 32768 * 128 * (64 + 2) * 4


def test_binding_refuses_what_32_bits_would_lose():
    torch = pytest.importorskip("torch")
    apart = torch.zeros(1).expand(1).as_strided((1, 4, 64), (256, 0, 0))
    far = torch.empty_strided((2, 4, 64), ((1 << 32) + 256, 64, 1), device="meta")
    near = torch.empty((2, 4, 64), device="meta")
    k = torch.empty((2, 2, 64), device="meta")
    cu = torch.empty(2, dtype=torch.int32, device="meta")
    for q, out in ((far, near), (near, far)):
        with pytest.raises(fvb.FlashVLAError, match="2\\^20"):
            fvb.prompt_attention(q, k, k, cu, cu, out)
    with pytest.raises(fvb.FlashVLAError, match="side by side"):
        fvb.prompt_attention(apart, apart, apart, cu, cu, apart)
    pool, refs = torch.zeros(2, 10, 2, 16, 64), torch.zeros(10, dtype=torch.int32)
    table, length = torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    c = fvb.PageCache(pool, pool.clone(), table, length, refs)
    q, k = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64)
    seqs, pos = torch.zeros(3, dtype=torch.int32), torch.zeros(1, 3, dtype=torch.int32)
    for layer in (2, -1, 1 << 32):
        with pytest.raises(fvb.FlashVLAError, match="layer"):
            c.attend(layer, q, seqs, q.clone())
        with pytest.raises(fvb.FlashVLAError, match="layer"):
            c.append(layer, q, k, k, pos, seqs, seqs, (32,))


@pytest.mark.parametrize("q_at,k_at,ldk", [(0, 496, 384), (64, 0, 384), (256, 240, 384), (272, 0, 384),
                                           (512, 384, 384), (0, 512, 392)])
def test_columns_of_one_matrix_that_overlap(q_at, k_at, ldk):
    """q_out (4 heads of 64) and k_out (2) from these bytes of one bf16 matrix on, rows of 384
    elements (768 bytes): columns apart would be taken, these are not."""
    a = rope_args(q_out=(P << 3) + q_at, k_out=(P << 3) + k_at, ldq_out=384, ldk_out=ldk)
    refused(fvb.lib().fv_rope_append(ctypes.byref(a), ctypes.byref(cache()), None), "overlap")


def test_binding_refuses_a_cache_elsewhere():
    torch = pytest.importorskip("torch")
    pool, refs = torch.zeros(2, 10, 2, 16, 64), torch.zeros(10, dtype=torch.int32)
    table, length = torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    c = fvb.PageCache(pool, pool.clone(), table, length, refs)
    q, k = (torch.empty((3, h, 64), device="meta") for h in (4, 2))
    seqs, pos = (torch.empty(s, dtype=torch.int32, device="meta") for s in ((3,), (1, 3)))
    with pytest.raises(fvb.FlashVLAError, match="the cache on cpu"):
        c.append(0, q, k, k, pos, seqs, seqs, (32,))


# Where the operands of rope_args begin; its rows of 256 (queries) and 128 (keys and values) bf16
Q, K, V, POOL = P, P << 1, P << 2, P << 6


@pytest.mark.parametrize("kw", [
    # queries in place, in a matrix that keys or values have a head of as well
    dict(q_out=Q, k=Q + 384), dict(q_out=Q, v=Q + 384), dict(q_out=Q, k=Q), dict(q_out=Q, k=Q + 384, k_out=None),
    # keys in place
    dict(k_out=K, q=K), dict(k_out=K, v=K + 128), dict(k_out=K, v=K),
    # both in place
    dict(q_out=Q, k=Q + 384, k_out=Q + 384), dict(q_out=Q, k=Q, k_out=Q),
    # columns of one packed matrix, the keys' one head too early
    dict(q_out=Q, ldq=512, ldq_out=512, k=Q + 384, k_out=Q + 384, ldk=512, ldk_out=512, v=Q + 768, ldv=512)],
    ids=str)
def test_rotation_in_place_over_other_operands(kw):
    a = rope_args(**kw)
    refused(fvb.lib().fv_rope_append(ctypes.byref(a), ctypes.byref(cache(k=POOL, v=POOL << 1)), None), "overlap")


def test_rotation_in_place_without_a_cache():
    a = rope_args(q_out=Q, k=Q + 384)
    refused(fvb.lib().fv_rope_append(ctypes.byref(a), None, None), "overlap")


# A layer of cache() has 10 pages of 2 heads, 16 rows of 64: 40960 bytes
LAYER = 10 * 2 * 16 * 64 * 2


@pytest.mark.parametrize("pool", ["k", "v"])
def test_outputs_in_the_pages(pool):
    L, ref = fvb.lib(), ctypes.byref
    n = ctypes.c_size_t()
    for layer, at in ((0, 0), (1, LAYER), (1, 2 * LAYER - 16)):
        inside = POOL + at
        c = cache(k=POOL << 1, v=POOL << 1)
        setattr(c, pool, POOL)
        for kw in (dict(q_out=inside), dict(k_out=inside)):
            refused(L.fv_rope_append(ref(rope_args(layer=layer, **kw)), ref(c), None), "pages")
        refused(L.fv_paged_attention(ref(paged_args(out=inside, layer=layer)), ref(c), None), "pages")
        for a, b in ((inside, P), (P, inside)):
            refused(L.fv_pages_gather(ref(c), P, 1, 5, a, b, None), "pages")
    # keys and values in one pool
    refused(L.fv_rope_append(ref(rope_args()), ref(cache(k=POOL, v=POOL)), None), "cache k and v")


def test_workspace_over_other_operands():
    L, ref = fvb.lib(), ctypes.byref
    c, n = cache(max_pages=4000, k=POOL, v=POOL << 1), ctypes.c_size_t()
    assert L.fv_paged_attention_workspace(ref(paged_args()), ref(c), ref(n)) == 0
    for work in (P, P << 1, POOL - 16, (POOL << 1) + LAYER - 16):
        refused(L.fv_paged_attention(ref(paged_args(work=work, work_bytes=n.value)), ref(c), None), "work")


def test_gathered_keys_over_gathered_values():
    L, c = fvb.lib(), cache(k=POOL, v=POOL << 1)
    out = 2 * 3 * 5 * 2 * 64 * 2  # bytes of 2 layers, 3 entries of 5 rows, 2 heads of 64
    for k, v in ((P, P), (P, P + out - 16), (P + out - 16, P)):
        refused(L.fv_pages_gather(ctypes.byref(c), P, 3, 5, k, v, None), "overlap")
    # sizes that 64 bits do not hold
    huge = cache(n_layers=1024, n_kv_heads=1024, head_dim=256, dtype=fvb.FV_FP32, k=POOL, v=POOL)
    refused(L.fv_pages_gather(ctypes.byref(huge), P, 65536, (1 << 31) - 1, P, P << 1, None), "overlap")


def test_binding_refuses_what_would_need_a_gradient():
    """The calls form none and write through pointers: in grad mode such tensors are refused, under
    no_grad they are taken (and then refused for not being on a GPU)."""
    torch = pytest.importorskip("torch")
    pool, refs = torch.zeros(2, 10, 2, 16, 64), torch.zeros(10, dtype=torch.int32)
    table, length = torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    seqs, pos = torch.zeros(3, dtype=torch.int32), torch.zeros(1, 3, dtype=torch.int32)
    cum = torch.tensor([0, 3], dtype=torch.int32)

    def calls(i):
        """Every call with its i-th floating tensor requiring a gradient."""
        def t(j, *shape):
            return torch.zeros(*shape, requires_grad=i == j)
        c = fvb.PageCache(t(9, 2, 10, 2, 16, 64), t(9, 2, 10, 2, 16, 64), table, length, refs)
        yield (0, 1), lambda: (fvb.PageCache(t(0, 2, 10, 2, 16, 64), t(1, 2, 10, 2, 16, 64), table, length, refs),
                               c.attend(0, t(9, 3, 4, 64), seqs, t(9, 3, 4, 64)))
        yield (0, 1, 2, 3), lambda: fvb.prompt_attention(t(0, 3, 4, 64), t(1, 3, 2, 64), t(2, 3, 2, 64), cum,
                                                         cum, t(3, 3, 4, 64))
        yield (0, 1, 2, 3), lambda: fvb.rope(t(0, 3, 4, 64), t(1, 3, 2, 64), pos, (32,), t(2, 3, 4, 64),
                                             t(3, 3, 2, 64))
        yield range(5), lambda: c.append(0, t(0, 3, 4, 64), t(1, 3, 2, 64), t(2, 3, 2, 64), pos, seqs, seqs,
                                         (32,), q_out=t(3, 3, 4, 64), k_out=t(4, 3, 2, 64))
        yield (0, 1), lambda: c.attend(0, t(0, 3, 4, 64), seqs, t(1, 3, 4, 64))
        yield (0, 1), lambda: c.gather(seqs, t(0, 2, 3, 5, 2, 64), t(1, 2, 3, 5, 2, 64))

    for i in range(5):
        for takes, call in calls(i):
            with pytest.raises(fvb.FlashVLAError, match="gradient" if i in takes else "GPU") as e:
                call()
            assert e.value.status == fvb.FV_ERR_INVALID_ARG
            with torch.no_grad(), pytest.raises(fvb.FlashVLAError, match="on a GPU"):
                call()
