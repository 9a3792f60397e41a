"""Operators of the observation context in 8 bits: what they compute, and the calls measured.

A cache of keys and values in e4m3 numbers, with a power of two as the scale of each block
(16 positions of one kv head):

  append  rotary positions on new queries and keys, and the new keys and values quantised into
          the pages of the cache
  read    sequences copied out of the pages, dense, as the action expert takes them
  attend  attention of one new token a sequence over the pages
  part    attention of several new tokens a sequence over the pages: parts of prompts, chunks

A case names its operator in `op`.  `run` computes the plain form from elementary torch
operations (own = False) or calls the framework (own = True).
"""
import math
import random

import numpy as np
import torch

own = False

# (query heads, kv heads, head dim): the pi0.5-shaped expert's (and its language model's), and
# the smaller and more finely grouped ones of the repository's tests.
_PI05 = dict(heads=8, kv=1, head_dim=256)
_GQA128 = dict(heads=32, kv=8, head_dim=128)
_GQA192 = dict(heads=4, kv=2, head_dim=192)
_MID64 = dict(heads=8, kv=2, head_dim=64)
_SHAPES = [_PI05, _PI05, _PI05, _GQA128, _GQA128, _GQA192, _MID64]

BLOCK = 16  # positions that share a scale


def _case(name, op, shape, seqs, lmin, lmax, dtype="bf16", page=16, **kw):
    c = dict(op=op, seqs=seqs, lmin=lmin, lmax=lmax, dtype=dtype, page=page, **shape)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One generated token for each of 64 robots, in blocks that are part-filled: latency.
        _case("append_token_b64", "append", _PI05, 64, 300, 816, nmin=1, nmax=1),
        # The observations of 64 robots, whole prompts, keys also kept dense for their own attention.
        _case("append_prompt_b64", "append", _PI05, 64, 300, 816, nmin=816, nmax=816),
        # Later parts of prompts, beginning and ending inside blocks, many kv heads.
        _case("append_parts_gqa128", "append", _GQA128, 48, 200, 2100, page=64, nmin=1, nmax=511),
        # The observations of 64 robots handed to the action expert, all layers: bandwidth.
        _case("read_b64", "read", _PI05, 64, 300, 816, layers=18),
        # One robot's observation, all layers: the smallest hand-over.
        _case("read_b1", "read", _PI05, 1, 560, 560, layers=18),
        # One robot's next token after a 3-view observation: latency.
        _case("attend_b1", "attend", _PI05, 1, 816, 816),
        # A server's next tokens over ragged observations.
        _case("attend_b64", "attend", _PI05, 64, 300, 816),
        # Long contexts, many kv heads, larger pages: bandwidth.
        _case("attend_long_b192", "attend", _GQA128, 192, 1, 8191, page=64),
        # A chunk of 50 new tokens after one robot's observation: latency.
        _case("part_b1", "part", _PI05, 1, 866, 866, nmin=50, nmax=50, causal=True),
        # A few new tokens for each of 64 ragged observations.
        _case("part_b64", "part", _PI05, 64, 300, 866, nmin=1, nmax=61, causal=True),
        # The last part of a long prompt (a video) over all that came before: arithmetic.
        _case("part_long", "part", _PI05, 1, 28672, 28672, nmin=4096, nmax=4096, causal=True),
        # fp32 queries and results, every key seen, odd lengths.
        _case("part_fp32", "part", _MID64, 5, 60, 1301, dtype="fp32", nmin=33, nmax=301, causal=False),
    ]


def _cost(c):
    """A rough time in us."""
    w = work(c)
    return 10.0 + w["bytes"] / 3e6 + w["flops"] / (5e8 if c["dtype"] == "bf16" else 1.5e8)


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["append", "append", "read", "attend", "attend", "part", "part"])
        dtype = "fp32" if rng.random() < 0.25 else "bf16"
        page = rng.choice([16, 16, 32, 48, 64, 128])
        seqs = spread(1, 256)
        lmax = spread(1, {"append": 4096, "read": 2048, "attend": 16384, "part": 20000}[op])
        lmin = lmax if rng.random() < 0.3 else rng.randint(1, lmax)
        kw = {}
        if op == "append":
            kw["nmax"] = rng.choice([1, lmax, spread(1, lmax)])
            kw["nmin"] = rng.choice([1, kw["nmax"]])
        elif op == "read":
            kw["layers"] = rng.randint(1, 18)
        elif op == "part":
            kw["nmax"] = spread(1, lmax)
            kw["nmin"] = rng.randint(1, kw["nmax"])
            kw["causal"] = rng.random() < 0.75
        c = _case(None, op, rng.choice(_SHAPES), seqs, lmin, lmax, dtype=dtype, page=page, **kw)
        # no more than the largest listed one, no more than 2 G values in a cache, and no more
        # than 1.2 G scores of padded rows in the plain form
        held = sum(_lengths(c)) * c["kv"] * c["head_dim"] * kw.get("layers", 1)
        scores = seqs * lmax * c["heads"] * kw.get("nmax", 1) if op in ("attend", "part") else 0
        if _cost(c) <= 2200.0 and held <= 1 << 31 and scores <= 1.2e9:
            return c


# ------------------------------------------------------------------ inputs

def _spread(lo, hi, count, at):
    n = [lo + int((at + b * 0.6180339887498949) % 1.0 * (hi - lo + 1)) for b in range(count)]
    n[-1] = hi
    return n


def _lengths(c):
    """Lengths spread over [lmin, lmax], a function of the case alone; the last is lmax."""
    return _spread(c["lmin"], c["lmax"], c["seqs"], 0.5)


def _new(c):
    """New tokens of each sequence, the last ones of its length."""
    return [min(n, m) for n, m in zip(_spread(c["nmin"], c["nmax"], c["seqs"], 0.3), _lengths(c))]


def _gen(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + tag) % (1 << 62))
    return g


def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _randn(c, seed, tag, *shape):
    return torch.randn(*shape, generator=_gen(seed, tag), device="cuda", dtype=_type(c))


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _sections(c):
    """Rotary pairs of time, height and width: a quarter and twice three eighths of them."""
    d = c["head_dim"]
    return (d // 8, 3 * d // 16, 3 * d // 16)


def _positions(n):
    """int [3, n] of a prompt: 16x16 views of images one after another, then text.  Views fill
    whole multiples of 256 tokens; the text goes on after the largest position so far."""
    j = np.arange(n)
    views = max(0, (n - 40) // 256)
    p = np.stack([j // 256, j // 16 % 16, j % 16])
    start = views + 16 if views else 0
    text = j >= 256 * views
    p[:, text] = start + (j[text] - 256 * views)
    return p


def _pool(c, lens, seed, layers=1):
    """A cache whose sequence b is the table's row b, its pages all over the pool.  Codes are what
    N(0, 1) values give: a block's largest is near 448, so the others have a deviation near 100,
    with scales around 2^-7."""
    pl = c["page"]
    need = [-(-n // pl) for n in lens]
    total = sum(need) + 8
    ids = np.random.default_rng(int(seed)).permutation(total)
    table = np.full((len(lens), max(need) + 2), -1, np.int64)
    first = np.cumsum([0] + need)
    for b, n in enumerate(need):
        table[b, :n] = ids[first[b]:first[b + 1]]
    refs = np.zeros(total, np.int64)
    refs[ids[:first[-1]]] = 1
    shape = (layers, total, c["kv"], pl, c["head_dim"])

    def codes(tag):
        x = torch.randn(shape, generator=_gen(seed, tag), device="cuda", dtype=torch.bfloat16) * 100
        return x.clamp_(-448, 448).to(torch.float8_e4m3fn)

    def scales(tag):
        b = torch.randint(119, 122, shape[:3] + (pl // BLOCK,), generator=_gen(seed, tag), device="cuda")
        return b.to(torch.uint8).view(torch.float8_e8m0fnu)

    return dict(k=codes(11), v=codes(12), k_scale=scales(13), v_scale=scales(14), table=_ints(table),
                len=_ints(lens), refs=_ints(refs))


def _cache(c, p):
    """The framework's cache over a pool's tensors."""
    from paper_2608_27384_amd.flashvla import QuantCache
    return QuantCache(p["k"], p["v"], p["k_scale"], p["v_scale"], p["table"], p["len"], p["refs"],
                      dtype=_type(c))


def prepare(case, seed):
    c = case
    lens = _lengths(c)
    H, G, D = c["heads"], c["kv"], c["head_dim"]
    p = _pool(c, lens, seed, c.get("layers", 1))
    s = dict(case=c, lens=lens, pool=p, cache=_cache(c, p) if own else None)
    if c["op"] == "append":
        # the packed product's output: queries, keys and values side by side in a row
        new = _new(c)
        at = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, new)])
        pos = np.concatenate([_positions(n)[:, n - m:] for n, m in zip(lens, new)], 1)
        qkv = _randn(c, seed, 1, len(at), H + 2 * G, D)
        dense = c["nmax"] > 1  # the keys are also kept dense
        s.update(q=qkv[:, :H], k=qkv[:, H:H + G], v=qkv[:, H + G:], pos=_ints(pos), at=_ints(at),
                 seqs=_ints(np.repeat(np.arange(len(lens)), new)),
                 axis=_ints(np.repeat(np.arange(3), _sections(c))),
                 q_out=torch.empty(len(at), H, D, dtype=_type(c), device="cuda"),
                 k_out=torch.empty(len(at), G, D, dtype=_type(c), device="cuda") if dense else None)
    elif c["op"] == "read":
        shape = (c["layers"], len(lens), max(lens), G, D)
        s.update(seqs=_ints(np.arange(len(lens))), k_out=_randn(c, seed, 4, *shape),
                 v_out=_randn(c, seed, 5, *shape))
    else:
        new = _new(c) if c["op"] == "part" else [1] * len(lens)
        s.update(q=_randn(c, seed, 1, sum(new), H, D), seqs=_ints(np.arange(len(lens))),
                 cu_q=_ints(np.cumsum([0] + new)), new=_ints(new), most=max(new),
                 out=torch.empty(sum(new), H, D, dtype=_type(c), device="cuda"))
    torch.cuda.synchronize()
    return s


# ------------------------------------------------------------------ one pass

def run(state):
    s = state
    return {"append": _run_append, "read": _run_read, "attend": _run_attend,
            "part": _run_attend}[s["case"]["op"]](s)


# A block of 16 positions of a head lies in memory as slabs of 64 elements.  Keys: [slab][position]
# [64].  Values: [slab][position / 4][element % 16][element % 64 / 16][position % 4], four positions
# side by side, as the matrix unit takes them.  Both as [..., positions, elements] here.

def _k_rows(x):
    *lead, pl, D = x.shape
    return x.reshape(*lead, pl // BLOCK, D // 64, BLOCK, 64).transpose(-3, -2).reshape(*lead, pl, D)


def _v_rows(x):
    *lead, pl, D = x.shape
    x = x.reshape(-1, pl // BLOCK, D // 64, 4, 16, 4, 4)
    return x.permute(0, 1, 3, 6, 2, 5, 4).reshape(*lead, pl, D)


def _k_stored(x):
    *lead, pl, D = x.shape
    return x.reshape(*lead, pl // BLOCK, BLOCK, D // 64, 64).transpose(-3, -2).reshape(*lead, pl, D)


def _v_stored(x):
    *lead, pl, D = x.shape
    x = x.reshape(-1, pl // BLOCK, 4, 4, D // 64, 4, 16)
    return x.permute(0, 1, 4, 2, 6, 5, 3).reshape(*lead, pl, D)


def _power(e):
    """2^e of whole numbers as fp32, exactly (2^-126 below that)."""
    return ((e.clamp(min=-126) + 127) << 23).to(torch.int32).view(torch.float32)


def _exponent(scale):
    return scale.view(torch.uint8).to(torch.int32) - 127


def _values(codes, scale, rows):
    """fp32 values of pages [..., page_len, D] with scales [..., page_len / 16]."""
    x = rows(codes.view(torch.uint8)).view(torch.float8_e4m3fn).float()
    return x * _power(_exponent(scale)).repeat_interleave(BLOCK, -1)[..., None]


def _encode(x):
    """e4m3 codes, to the nearest (ties to even), saturating; what is not finite becomes NaN."""
    c = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return torch.where(x.isfinite(), c, torch.full_like(c, 0x7f))


def _write(s, x, codes, scale, rows, stored):
    """The tokens' fp32 rows x [n, G, D] into one layer's pages.  A block that is written from its
    first row on starts anew (its other rows become zeros); one that is written from another row on
    keeps its scale where that is the larger, or its rows are rounded again."""
    c, table = s["case"], s["pool"]["table"]
    pl = c["page"]
    at, seqs = s["at"].long(), s["seqs"].long()
    page = table[seqs, at // pl].long()
    block, place = torch.unique(page * (pl // BLOCK) + at % pl // BLOCK, return_inverse=True)
    n, G, D = x.shape
    first = torch.full_like(block, BLOCK).scatter_reduce(0, place, at % BLOCK, "amin")
    size = torch.where(x.isfinite(), x.abs(), torch.zeros_like(x)).amax(-1)
    top = size.new_zeros(len(block), G).scatter_reduce(0, place[:, None].expand(-1, G), size, "amax")
    m, k = torch.frexp(top)  # m in [0.5, 1)
    e = torch.where(m <= 0.875, k - 9, k - 8)
    e = torch.where(top > 0, e, torch.full_like(e, -117)).clamp(-117, 119)
    keeps = (first > 0)[:, None]
    # [pages, G, blocks of a page, ...] by blocks
    per, b = pl // BLOCK, block % (pl // BLOCK)
    old_e = _exponent(scale)[block // per, :, b]
    now = torch.where(keeps, torch.maximum(e, old_e), e)
    old = codes.view(torch.uint8).reshape(codes.shape[0], G, per, BLOCK, D)[block // per, :, b]
    old = rows(old).view(torch.float8_e4m3fn).float()
    again = old * _power(old_e - now)[..., None, None]
    again = torch.where(keeps[..., None, None], again, torch.zeros_like(again))
    again[place, :, at % BLOCK] = x * _power(-now)[place][..., None]
    codes.view(torch.uint8).view(codes.shape[0], G, per, BLOCK, D)[block // per, :, b] = stored(_encode(again))
    scale.view(torch.uint8)[block // per, :, b] = (now + 127).to(torch.uint8)


def _run_append(s):
    c, p = s["case"], s["pool"]
    out = {"q": s["q_out"], "k": s["k_out"], "k_pages": p["k"], "v_pages": p["v"],
           "k_scale": p["k_scale"], "v_scale": p["v_scale"]}
    if own:
        s["cache"].append(0, s["q"], s["k"], s["v"], s["pos"], s["seqs"], s["at"], _sections(c),
                          theta=1e4, q_out=s["q_out"], k_out=s["k_out"])
        return out
    D = c["head_dim"]
    inv = 1e4 ** (-torch.arange(D // 2, dtype=torch.float64, device="cuda") * 2.0 / D)
    ang = s["pos"][s["axis"]].double().t() * inv  # 64 bits: far positions turn many times
    cos, sin = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]

    def turn(x):
        a, b = x.float()[..., :D // 2], x.float()[..., D // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    k = turn(s["k"])
    s["q_out"].copy_(turn(s["q"]))
    if s["k_out"] is not None:
        s["k_out"].copy_(k)
    _write(s, k, p["k"][0], p["k_scale"][0], _k_rows, _k_stored)
    _write(s, s["v"].float(), p["v"][0], p["v_scale"][0], _v_rows, _v_stored)
    return out


def _run_read(s):
    c, p = s["case"], s["pool"]
    if own:
        s["cache"].gather(s["seqs"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    k_out, v_out = s["k_out"], s["v_out"]
    seqs, ld = s["seqs"].long(), k_out.shape[2]
    table = p["table"][seqs, :-(-ld // c["page"])].clamp(min=0).long()
    live = (torch.arange(ld, device="cuda")[None] < p["len"][seqs][:, None])[None, :, :, None, None]

    def dense(codes, scale, rows, dst):  # [layers, entries, pages, G, page_len, D] to rows
        x = _values(codes[:, table], scale[:, table], rows).transpose(3, 4)
        x = x.reshape(dst.shape[0], len(seqs), -1, *dst.shape[3:])[:, :, :ld]
        dst.copy_(torch.where(live, x.to(dst.dtype), dst))

    dense(p["k"], p["k_scale"].view(torch.uint8), _k_rows, k_out)
    dense(p["v"], p["v_scale"].view(torch.uint8), _v_rows, v_out)
    return {"k": k_out, "v": v_out}


def _run_attend(s):
    c, p = s["case"], s["pool"]
    one = c["op"] == "attend"
    if own:
        if one:
            s["cache"].attend(0, s["q"], s["seqs"], s["out"], max_len=max(s["lens"]))
        else:
            s["cache"].attend_part(0, s["q"], s["cu_q"], s["seqs"], s["out"], causal=c["causal"],
                                   max_len=max(s["lens"]))
        return s["out"]
    H, G, D, pl = c["heads"], c["kv"], c["head_dim"], c["page"]
    n, most, wide = len(s["lens"]), s["most"], -(-max(s["lens"]) // c["page"])
    seqs = s["seqs"].long()
    table = p["table"][seqs, :wide].clamp(min=0).long()

    def dense(codes, scale, rows):
        x = _values(codes[0][table], scale.view(torch.uint8)[0][table], rows)
        return x.transpose(1, 2).reshape(n, G, wide * pl, D)

    k, v = dense(p["k"], p["k_scale"], _k_rows), dense(p["v"], p["v_scale"], _v_rows)
    # queries as [sequences, most, ...], a row's place in the packed ones beside it
    i = torch.arange(most, device="cuda")
    place = s["cu_q"][:-1].long()[:, None] + i
    here = i < s["new"][:, None]
    q = s["q"][place.clamp(max=len(s["q"]) - 1)].float()
    q = q.reshape(n, most, G, H // G, D).transpose(1, 2).reshape(n, G, most * (H // G), D)
    x = ((q @ k.transpose(2, 3).contiguous()) / math.sqrt(D)).reshape(n, G, most, H // G, wide * pl)
    j = torch.arange(wide * pl, device="cuda")
    sees = p["len"][seqs][:, None].expand(n, most)
    if not one and c["causal"]:
        sees = sees - s["new"][:, None] + i + 1
    x.masked_fill_((j >= sees[..., None])[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    e = x.sub_(torch.where(top.isfinite(), top, torch.zeros_like(top))).exp_()
    total = e.sum(-1, keepdim=True)
    o = (e.reshape(n, G, -1, wide * pl) @ v).reshape(n, G, most, H // G, D) / total
    s["out"].copy_(o.transpose(1, 2).reshape(n, most, H, D)[here])
    return s["out"]


# ------------------------------------------------------------------ work

def _pairs(c):
    lens = _lengths(c)
    if c["op"] == "attend":
        return sum(lens)
    return sum(m * n - (m * (m - 1) // 2 if c["causal"] else 0) for m, n in zip(_new(c), lens))


def work(case):
    c = case
    H, G, D, pl = c["heads"], c["kv"], c["head_dim"], c["page"]
    e = 2 if c["dtype"] == "bf16" else 4
    lens = _lengths(c)
    blocks = sum(-(-n // BLOCK) for n in lens)
    if c["op"] == "append":
        new = _new(c)
        n = sum(new)
        wrote = sum(-(-a // BLOCK) - (a - b) // BLOCK for a, b in zip(lens, new))
        dense = G if c["nmax"] > 1 else 0
        return {"bytes": n * (D * (e * (2 * H + 2 * G + dense) + 2 * G) + 4 * 5) + wrote * 2 * G,
                "flops": 3 * n * (H + G) * D}
    if c["op"] == "read":
        L, n = c["layers"], sum(lens)
        return {"bytes": 2 * L * G * (n * D * (1 + e) + blocks) + 4 * sum(-(-x // pl) for x in lens),
                "flops": 2 * L * G * n * D}
    rows = len(lens) if c["op"] == "attend" else sum(_new(c))
    return {"bytes": 2 * G * (D * sum(lens) + blocks) + 2 * rows * H * D * e + 4 * sum(-(-x // pl) for x in lens),
            "flops": 4 * D * H * _pairs(c)}


# ------------------------------------------------------------------ exact

def _e4m3_numbers():
    """The 256 numbers of e4m3: sign, 4 bits of exponent (bias 7), 3 of mantissa; 127 is NaN."""
    t = []
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        x = math.nan if b & 127 == 127 else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        t.append(-x if b >= 128 else x)
    return torch.tensor(t, dtype=torch.float64, device="cuda")


def _byte_of(D, values):
    """Where in a block's bytes the element (position, d) lies: [16, D]."""
    t, d = torch.arange(16, device="cuda")[:, None], torch.arange(D, device="cuda")[None]
    if values:
        return d // 64 * 1024 + t // 4 * 256 + d % 16 * 16 + d % 64 // 16 * 4 + t % 4
    return d // 64 * 1024 + t * 64 + d % 64


def _nearest(y):
    """y to e4m3 in 64 bits: steps of 2^-9 below 2^-6, of an eighth of the leading power above."""
    size = y.abs().clamp(2.0 ** -6, 448.0)
    step = torch.exp2(torch.floor(torch.log2(size)) - 3)
    return (torch.round(y / step) * step).clamp(-448.0, 448.0)


def _exact_pages(s, x, codes, scale, values):
    """Codes (as numbers) and scales of layer 0 after rows x [n, G, D] in 64 bits were written."""
    c = s["case"]
    pl, D, G = c["page"], c["head_dim"], c["kv"]
    num = _e4m3_numbers()[codes[0].view(torch.uint8).long()]
    P = num.shape[0]
    flat = num.reshape(P * G * (pl // 16), 16 * D)
    power = torch.exp2(scale[0].view(torch.uint8).double() - 127).reshape(-1).clone()
    at, seqs = s["at"].long(), s["seqs"].long()
    page = s["pool"]["table"].long()[seqs, at // pl]
    heads = torch.arange(G, device="cuda")[None]
    block = (page[:, None] * G + heads) * (pl // 16) + (at % pl // 16)[:, None]  # [n, G]
    top = torch.zeros(len(power), dtype=torch.float64, device="cuda")
    top.scatter_reduce_(0, block.reshape(-1), x.abs().amax(-1).reshape(-1), "amax")
    starts = torch.zeros(len(power), dtype=torch.bool, device="cuda")
    starts[block[at % 16 == 0].reshape(-1)] = True
    hit = torch.unique(block)
    want = torch.exp2(torch.ceil(torch.log2(top[hit].clamp(min=2.0 ** -109) / 448.0)).clamp(-117, 119))
    old = torch.where(starts[hit], torch.zeros_like(want), power[hit])
    power[hit] = torch.maximum(want, old)
    flat[hit] = _nearest(flat[hit] * (old / power[hit])[:, None])
    where = _byte_of(D, values)[at % 16]  # [n, D]
    flat[block[..., None], where[:, None].expand(-1, G, -1)] = _nearest(x / power[block][..., None])
    return flat.reshape(1, *num.shape), power.reshape(scale.shape)


def _exact_rows(s, codes, scale, layer, b, n, g, values):
    """Positions 0..n of sequence b, kv head g: [n, D] in 64 bits."""
    c = s["case"]
    ids = s["pool"]["table"][b, :-(-n // c["page"])].long()
    D = c["head_dim"]
    num = _e4m3_numbers()[codes[layer, ids, g].view(torch.uint8).long()].reshape(-1, 16 * D)
    num = num[:, _byte_of(D, values).reshape(-1)].reshape(-1, 16, D)
    power = torch.exp2(scale[layer].view(torch.uint8)[ids, g].double() - 127).reshape(-1)
    return (num * power[:, None, None]).reshape(-1, D)[:n]


def exact(case, seed):
    c = case
    D, H, G = c["head_dim"], c["heads"], c["kv"]
    s = prepare(c, seed)
    p = s["pool"]
    if c["op"] == "append":
        half = D // 2
        th = torch.empty(s["pos"].shape[1], half, dtype=torch.float64, device="cuda")
        i = 0
        for a, width in enumerate(_sections(c)):
            for _ in range(width):
                th[:, i] = s["pos"][a].double() * math.pow(1e4, -2.0 * i / D)
                i += 1
        z = torch.polar(torch.ones_like(th), th)[:, None]  # a pair is a complex number, turned by z

        def turned(x):
            w = torch.complex(x[..., :half].double(), x[..., half:].double()) * z
            return torch.cat([w.real, w.imag], -1)

        k = turned(s["k"])
        kp, ks = _exact_pages(s, k, p["k"], p["k_scale"], False)
        vp, vs = _exact_pages(s, s["v"].double(), p["v"], p["v_scale"], True)
        return {"q": turned(s["q"]), "k": k if s["k_out"] is not None else None, "k_pages": kp,
                "v_pages": vp, "k_scale": ks, "v_scale": vs}
    if c["op"] == "read":
        if c["layers"] * c["seqs"] * G > 6000:
            return None
        out = {}
        for name in ("k", "v"):
            x = s[name + "_out"].double()
            for layer in range(c["layers"]):
                for b, n in enumerate(s["lens"]):
                    for g in range(G):
                        x[layer, b, :n, g] = _exact_rows(s, p[name], p[name + "_scale"], layer, b, n, g,
                                                         name == "v")
            out[name] = x
        return out
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    cq = s["cu_q"].tolist()
    for b, n in enumerate(s["lens"]):
        m = cq[b + 1] - cq[b]
        for g in range(G):
            keys = _exact_rows(s, p["k"], p["k_scale"], 0, b, n, g, False)
            vals = _exact_rows(s, p["v"], p["v_scale"], 0, b, n, g, True)
            for h in range(g * H // G, (g + 1) * H // G):
                x = s["q"][cq[b]:cq[b + 1], h].double() @ keys.t() * D ** -0.5
                if c["op"] == "part" and c["causal"]:
                    x += torch.full_like(x, -math.inf).triu(n - m + 1)
                out[cq[b]:cq[b + 1], h] = torch.softmax(x, -1) @ vals
    return out


def _selfcheck():
    """Prints the listed cases' sizes and some drawn ones' (no GPU needed)."""
    rng = random.Random(0)
    for c in listed() + [draw(rng) for _ in range(16)]:
        print(c, work(c), round(_cost(c)))


if __name__ == "__main__":
    _selfcheck()
