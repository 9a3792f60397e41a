"""What the operators of the cache in 8 bits refuse: at the C boundary from the arguments alone (no
GPU is touched), and in the binding from the tensors' shapes, types and strides; the launch rules."""
import ctypes

import pytest

from paper_2608_27384_amd import flashvla as fvb
from test_context_refusals import P, paged_args, refused, rope_args

POOL = P << 8
LAYER = 10 * 2 * 16 * 64  # codes of a layer of cache(): 10 pages of 2 heads, 16 positions of 64


def cache(**kw):
    c = fvb.FvQuantPages(fvb.FV_BF16, 2, 2, 64, 16, 10, 4, 3, POOL, POOL << 1, POOL << 2, POOL << 3, P, P, P)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def part_args(**kw):
    a = fvb.FvPartArgs(P, P << 1, 256, 256, P, P, 2, 9, 4, 0, 0, 1, 0.125, None, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def test_structures_match_the_header():
    assert ctypes.sizeof(fvb.FvQuantPages) == 32 + 7 * 8
    assert ctypes.sizeof(fvb.FvPartArgs) == 16 + 8 + 16 + 6 * 4 + 4 + 4 + 8 + 8


@pytest.mark.parametrize("field,value", [
    ("dtype", 2), ("dtype", -1), ("n_layers", 0), ("n_layers", 1025), ("n_kv_heads", 0), ("head_dim", 80),
    ("page_len", 8), ("page_len", 24), ("page_len", 272), ("n_pages", 0), ("n_pages", (1 << 20) + 1),
    ("max_seqs", 0), ("max_seqs", 65537), ("max_pages", 0), ("max_pages", 65537), ("k", None), ("v", P + 8),
    ("k_scale", None), ("v_scale", None), ("table", None), ("len", P + 2), ("refs", None)])
def test_caches(field, value):
    L, c = fvb.lib(), cache(**{field: value})
    b, n = ctypes.byref(c), ctypes.c_size_t()
    refused(L.fv_quant_workspace(b, ctypes.byref(n)))
    refused(L.fv_quant_grow(b, P, P, 1, P, P, None))
    refused(L.fv_quant_fork(b, P, P, 1, P, P, None))
    refused(L.fv_quant_free(b, P, 1, P, None))
    refused(L.fv_quant_compact(b, P, P, None))
    refused(L.fv_quant_gather(b, P, 1, 5, P, P << 1, None))
    refused(L.fv_quant_append(ctypes.byref(rope_args()), b, None))
    refused(L.fv_quant_attention(ctypes.byref(paged_args()), b, None))
    refused(L.fv_quant_attention_workspace(ctypes.byref(paged_args()), b, ctypes.byref(n)))
    refused(L.fv_quant_part_attention(ctypes.byref(part_args()), b, None))
    refused(L.fv_quant_part_workspace(ctypes.byref(part_args()), b, ctypes.byref(n)))


@pytest.mark.parametrize("kw", [
    dict(dtype=3), dict(dtype=fvb.FV_FP32), dict(head_dim=128), dict(n_q_heads=3), dict(n=-1), dict(n=(1 << 26) + 1),
    dict(n_axes=0), dict(n_axes=5), dict(sections=(ctypes.c_int32 * 4)(8, 12, 11)), dict(theta=0.0),
    dict(layer=2), dict(layer=-1), dict(q=None), dict(k=P + 4), dict(v=None), dict(q_out=None), dict(ldq=255),
    dict(ldv=(1 << 20) + 8), dict(ldk_out=64), dict(pos=None), dict(seqs=None), dict(at=P + 1), dict(q_out=P + 64),
    dict(q_out=P << 1), dict(k_out=P << 2), dict(k_out=P << 3)], ids=str)
def test_append(kw):
    refused(fvb.lib().fv_quant_append(ctypes.byref(rope_args(**kw)), ctypes.byref(cache()), None))


def test_append_needs_a_cache_and_arguments():
    L = fvb.lib()
    refused(L.fv_quant_append(ctypes.byref(rope_args()), None, None), "NULL")
    refused(L.fv_quant_append(None, ctypes.byref(cache()), None), "NULL")
    assert L.fv_quant_append(ctypes.byref(rope_args(n=0, q=None)), ctypes.byref(cache()), None) == 0


@pytest.mark.parametrize("kw", [
    dict(n=-1), dict(n=65537), dict(n_q_heads=3), dict(max_len=-1), dict(layer=2), dict(scale=0.0),
    dict(scale=float("nan")), dict(q=None), dict(out=P + 8), dict(out=P + 512), dict(ldq=128), dict(ldo=260),
    dict(seqs=None)], ids=str)
def test_tokens(kw):
    refused(fvb.lib().fv_quant_attention(ctypes.byref(paged_args(**kw)), ctypes.byref(cache()), None))


@pytest.mark.parametrize("kw", [
    dict(n_seqs=-1), dict(n_seqs=65537), dict(n_q=-1), dict(n_q=(1 << 26) + 1), dict(n_q_heads=3), dict(n_q_heads=0),
    dict(max_len=-1), dict(layer=2), dict(layer=-1), dict(causal=2), dict(scale=0.0), dict(scale=-1.0),
    dict(scale=float("inf")), dict(q=None), dict(out=P + 8), dict(out=P + 512), dict(ldq=128), dict(ldo=260),
    dict(cu_q=None), dict(cu_q=P + 2), dict(seqs=None)], ids=str)
def test_parts(kw):
    refused(fvb.lib().fv_quant_part_attention(ctypes.byref(part_args(**kw)), ctypes.byref(cache()), None))


def test_nothing_to_do_touches_no_gpu():
    L, ref, c = fvb.lib(), ctypes.byref, cache()
    assert L.fv_quant_part_attention(ref(part_args(n_q=0, q=None)), ref(c), None) == 0
    assert L.fv_quant_part_attention(ref(part_args(n_seqs=0, q=None)), ref(c), None) == 0
    assert L.fv_quant_attention(ref(paged_args(n=0)), ref(c), None) == 0
    assert L.fv_quant_gather(ref(c), None, 0, 5, None, None, None) == 0
    assert L.fv_context_error() == b""


def test_outputs_in_the_cache():
    """Codes and scales of the layer: no result, workspace or kept key may lie there."""
    L, ref, n = fvb.lib(), ctypes.byref, ctypes.c_size_t()
    for i, name in enumerate(("k", "v", "k_scale", "v_scale")):
        layer = LAYER if i < 2 else 20
        for l in (0, 1):
            base = POOL << i
            for at in (base + l * layer, base + (l + 1) * layer - 1):
                at &= ~15
                for kw in (dict(q_out=at), dict(k_out=at)):
                    refused(L.fv_quant_append(ref(rope_args(layer=l, **kw)), ref(cache()), None), "pages")
                refused(L.fv_quant_attention(ref(paged_args(out=at, layer=l)), ref(cache()), None), "pages")
                refused(L.fv_quant_part_attention(ref(part_args(out=at, layer=l)), ref(cache()), None), "pages")
                for a, b in ((at, P), (P, at)):
                    refused(L.fv_quant_gather(ref(cache()), P, 1, 5, a, b, None), "pages")
    for kw in (dict(v=POOL), dict(k_scale=POOL + 100), dict(v_scale=POOL << 2)):
        refused(L.fv_quant_append(ref(rope_args()), ref(cache(**kw)), None), "overlap")
    refused(L.fv_quant_gather(ref(cache()), P, 1, 5, P, P, None), "overlap")


def test_workspaces():
    L, ref, n = fvb.lib(), ctypes.byref, ctypes.c_size_t()
    c = cache(max_pages=4000)
    for call, need, args in ((L.fv_quant_attention, L.fv_quant_attention_workspace, paged_args),
                             (L.fv_quant_part_attention, L.fv_quant_part_workspace, part_args)):
        assert need(ref(args()), ref(c), ref(n)) == 0 and n.value > 0
        refused(call(ref(args()), ref(c), None), "work")
        refused(call(ref(args(work=P << 4, work_bytes=n.value - 1)), ref(c), None), "work")
        refused(call(ref(args(work=(P << 4) + 8, work_bytes=n.value)), ref(c), None), "work")
        for work in (P, P << 1, POOL, POOL << 1, (POOL << 1) + LAYER - 16, POOL << 3):
            refused(call(ref(args(work=work, work_bytes=n.value)), ref(c), None), "work")


def test_lists():
    L, c = fvb.lib(), cache()
    b = ctypes.byref(c)
    for n in (-1, 5):
        refused(L.fv_quant_grow(b, P, P, n, P, P, None))
        refused(L.fv_quant_fork(b, P, P, n, P, P, None))
        refused(L.fv_quant_free(b, P, n, P, None))
    refused(L.fv_quant_grow(b, P, None, 1, P, P, None))
    refused(L.fv_quant_grow(b, P, P, 1, P, P + 4, None))
    refused(L.fv_quant_fork(b, None, P, 1, P, P, None))
    refused(L.fv_quant_free(b, P + 1, 1, P, None))
    refused(L.fv_quant_compact(b, None, P, None))
    refused(L.fv_quant_compact(b, P, None, None))
    refused(L.fv_quant_gather(b, P, -1, 5, P, P << 1, None))
    refused(L.fv_quant_gather(b, P, 65537, 5, P, P << 1, None))
    refused(L.fv_quant_gather(b, P, 1, -5, P, P << 1, None))
    refused(L.fv_quant_gather(b, P, 1, 5, P + 8, P << 1, None))


def tensors(**kw):
    torch = pytest.importorskip("torch")
    t = dict(k=torch.zeros(2, 10, 2, 32, 64).to(torch.float8_e4m3fn), v=torch.zeros(2, 10, 2, 32, 64).to(torch.float8_e4m3fn),
             k_scale=torch.zeros(2, 10, 2, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu),
             v_scale=torch.zeros(2, 10, 2, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu),
             table=torch.zeros(4, 3, dtype=torch.int32), length=torch.zeros(4, dtype=torch.int32),
             refs=torch.zeros(10, dtype=torch.int32))
    t.update(kw)
    return t


def test_binding_refuses_tensors():
    torch = pytest.importorskip("torch")

    def no(fn, *a, **kw):
        with pytest.raises(fvb.FlashVLAError) as e:
            fn(*a, **kw)
        assert e.value.status == fvb.FV_ERR_INVALID_ARG

    t = tensors()
    for kw in (dict(k=t["k"].view(torch.uint8)), dict(v=t["v"][:1]), dict(v=t["v"].view(torch.uint8)),
               dict(k_scale=t["k_scale"].view(torch.uint8)), dict(v_scale=t["v_scale"][..., :1]),
               dict(k_scale=t["k_scale"].transpose(0, 1)), dict(table=t["table"].long()),
               dict(length=t["length"][:3]), dict(refs=t["refs"][:9]), dict(dtype=torch.float16),
               dict(k=t["k"][..., 0]), dict(k=t["k"].transpose(2, 3))):
        no(fvb.QuantCache, **tensors(**kw))
    c = fvb.QuantCache(**t, dtype=torch.float32)
    q, k = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64)
    seqs, cum, pos = (torch.zeros(s, dtype=torch.int32) for s in ((3,), (4,), (1, 3)))
    no(c.attend, 0, q, seqs, q.clone())  # not on a GPU
    no(c.attend, 0, q.bfloat16(), seqs, q.bfloat16())
    no(c.attend_part, 0, q, cum, seqs, q.clone())
    no(c.attend_part, 0, q.bfloat16(), cum, seqs, q.bfloat16())
    no(c.attend_part, 0, q, cum, seqs[:2], q.clone())
    no(c.attend_part, 0, q, cum[:0], seqs, q.clone())
    no(c.attend_part, 0, q, cum[None], seqs, q.clone())
    no(c.attend_part, 0, q, cum.long(), seqs, q.clone())
    no(c.attend_part, 0, q[..., :32], cum, seqs, q[..., :32])
    no(c.attend_part, 0, q, cum, seqs, q[:2])
    for layer in (2, -1, 1 << 32):
        no(c.attend_part, layer, q, cum, seqs, q.clone())
    no(c.append, 0, q, k, None, pos, seqs, seqs, (32,))
    no(c.append, 0, q, k, k, pos, seqs, seqs, (32,))
    no(c.grow, seqs, seqs)
    no(c.gather, seqs, torch.zeros(2, 3, 5, 2, 64).bfloat16(), torch.zeros(2, 3, 5, 2, 64).bfloat16())
    no(c.gather, seqs, torch.zeros(2, 3, 5, 2, 64), torch.zeros(2, 3, 6, 2, 64))
    need = q.clone().requires_grad_()
    with pytest.raises(fvb.FlashVLAError, match="gradient"):
        c.attend_part(0, need, cum, seqs, q.clone())
    with torch.no_grad(), pytest.raises(fvb.FlashVLAError, match="on a GPU"):
        c.attend_part(0, need, cum, seqs, q.clone())


def part_plan(n_q, n_seqs, heads, kv, D, keys, dtype=fvb.FV_BF16):
    class Plan(ctypes.Structure):
        _fields_ = [("rows", ctypes.c_int32), ("chunk", ctypes.c_int32), ("n_chunks", ctypes.c_int32),
                    ("work_bytes", ctypes.c_size_t)]
    f = getattr(fvb.lib(), "_ZN2fv9plan_partERK12fv_part_argsRK14fv_quant_pagesi")
    f.restype, f.argtypes = Plan, [ctypes.POINTER(fvb.FvPartArgs), ctypes.POINTER(fvb.FvQuantPages), ctypes.c_int]
    a = part_args(n_q=n_q, n_seqs=n_seqs, n_q_heads=heads)
    c = cache(dtype=dtype, n_kv_heads=kv, head_dim=D)
    return f(ctypes.byref(a), ctypes.byref(c), keys)


@pytest.mark.parametrize("dtype", [fvb.FV_BF16, fvb.FV_FP32])
@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 1), (32, 8), (64, 64), (1024, 1), (1024, 1024)])
def test_every_part_is_a_launch(heads, kv, D, dtype):
    """Grids of less than 2^32 threads, of the row tiles by chunks and of the join, and chunks that
    cover the keys."""
    for n_q in (1, 50, 4096, (1 << 22) // heads, (1 << 28) // heads):
        for n_seqs in (1, 64, 65536):
            if n_seqs * kv > 1 << 22:
                continue
            for keys in (1, 16, 816, 28672, 1 << 24):
                p = part_plan(n_q, n_seqs, heads, kv, D, keys, dtype)
                tiles = (n_q * (heads // kv) // p.rows + n_seqs) * kv
                assert p.rows in (32, 64, 128) and tiles * p.n_chunks * 256 < 1 << 32
                assert p.n_chunks >= 1 and p.chunk % 32 == 0
                if p.n_chunks > 1:
                    assert n_q * heads * 512 < 1 << 32
                    assert p.work_bytes >= n_q * heads * p.n_chunks * (D + 2) * 4
                else:
                    assert p.work_bytes == 0


@pytest.mark.parametrize("n_q,n_seqs,heads,kv,D,keys,dtype,rows,chunk,chunks", [
    (50, 1, 8, 1, 256, 866, fvb.FV_BF16, 32, 128, 7),       # every wave of a chunk has one step
    (1982, 64, 8, 1, 256, 866, fvb.FV_BF16, 64, 896, 1),
    (6400, 128, 8, 1, 256, 866, fvb.FV_BF16, 128, 896, 1),
    (500, 1, 8, 1, 256, 8000, fvb.FV_BF16, 64, 1344, 6),
    (4096, 1, 8, 1, 256, 28672, fvb.FV_BF16, 128, 14336, 2),  # two workgroups a CU
    (4000, 8, 32, 8, 128, 2000, fvb.FV_BF16, 128, 2016, 1),
    (800, 5, 8, 2, 64, 1301, fvb.FV_FP32, 32, 1408, 1),
    (50, 1, 8, 1, 256, 900, fvb.FV_FP32, 32, 128, 8),
    (12800, 256, 8, 1, 256, 866, fvb.FV_FP32, 128, 896, 1),
    (1, 1, 8, 1, 256, 1 << 24, fvb.FV_BF16, 32, 1 << 19, 32)])
def test_parts_are_shared_out(n_q, n_seqs, heads, kv, D, keys, dtype, rows, chunk, chunks):
    p = part_plan(n_q, n_seqs, heads, kv, D, keys, dtype)
    assert (p.rows, p.chunk, p.n_chunks) == (rows, chunk, chunks)


def token_plan(n, heads, kv, D, keys, bf16):
    class Plan(ctypes.Structure):
        _fields_ = [("keys", ctypes.c_int32), ("chunk", ctypes.c_int32), ("n_chunks", ctypes.c_int32),
                    ("work_bytes", ctypes.c_size_t)]
    f = fvb.lib()._ZN2fv10plan_quantEiiiiib
    f.restype, f.argtypes = Plan, [ctypes.c_int] * 5 + [ctypes.c_bool]
    return f(n, heads, kv, D, keys, bf16)


def test_tokens_are_shared_out():
    """One chunk up to a length that grows with the workgroups of one chunk."""
    for n, heads, kv, D, bf16, most in ((1, 8, 1, 256, True, 448), (1, 8, 1, 256, False, 256), (2, 4, 2, 128, False, 448),
                                        (64, 8, 1, 256, True, 768), (64, 8, 1, 256, False, 256), (127, 8, 1, 64, True, 1524),
                                        (128, 8, 1, 256, True, 2048), (32, 32, 4, 128, False, 2048), (1, 128, 1, 64, True, 448),
                                        (16, 128, 1, 64, True, 2048), (4096, 8, 8, 64, True, 2048)):
        p, more = token_plan(n, heads, kv, D, most, bf16), token_plan(n, heads, kv, D, most + 1, bf16)
        assert p.n_chunks == 1 and p.work_bytes == 0
        assert more.n_chunks > 1 and more.work_bytes == n * more.n_chunks * heads * (D + 2) * 4


def test_tokens_of_an_append_are_shared_out():
    class Share(ctypes.Structure):
        _fields_ = [("tokens", ctypes.c_int32), ("parts", ctypes.c_int32)]
    f = fvb.lib()._ZN2fv11quant_shareEii
    f.restype, f.argtypes = Share, [ctypes.c_int] * 2
    for n, kv, tokens, parts in ((1, 1, 1, 1), (127, 1, 1, 1), (128, 1, 4, 4), (1023, 1, 4, 2), (1024, 1, 8, 4), (4096, 1, 8, 1),
                                 (1, 8, 1, 8), (127, 8, 1, 8), (128, 8, 4, 32), (1023, 8, 4, 4), (1024, 8, 8, 8),
                                 (4096, 8, 8, 2), (4104, 8, 8, 1), (512, 2, 4, 6), (1 << 26, 1024, 8, 1)):
        s = f(n, kv)
        assert (s.tokens, s.parts) == (tokens, parts), n
        wide = min(-(-n // tokens), 1 << 20)
        assert wide * 256 < 1 << 32 and -(-n // tokens // wide) < 1 << 16
    assert max(f(n, 1024).parts for n in range(1, 2000)) < 1 << 16
