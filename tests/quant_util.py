"""The cache in 8 bits by its definition, in 64 bits, and caches to test with.

A block is 16 positions of a kv head; a code is one of e4m3's numbers, worth itself times
2^(b - 127) with the block's scale byte b.  Quantising rounds to the nearest number, ties to the
even code, so a stored value is off by at most half a step: 2^-4 of it, or 2^-10 of the scale
where the number is below 2^-6 (steps of 2^-9)."""
import numpy as np

import context_util as cu


def _numbers():
    """What the 256 codes stand for: sign, exponent of 4 bits (bias 7), 3 bits; 127 is NaN."""
    x = []
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        v = np.nan if b & 127 == 127 else (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
        x.append(-v if b >= 128 else v)
    return np.array(x)


NUMBERS = _numbers()


def nearest(y):
    """Codes (uint8) of 64-bit numbers within +-448; NaN where they are not finite."""
    torch = cu.torch_mod()
    pos = torch.from_numpy(NUMBERS[:127]).to(y.device)
    mids = (pos[:-1] + pos[1:]) / 2  # exact
    a = y.abs().clamp(max=448.0).nan_to_num(0.0).contiguous()
    c = torch.bucketize(a, mids)  # the first midpoint that is not below: ties to the lower code
    tie = (c < 126) & (mids[c.clamp(max=125)] == a)
    c = torch.where(tie & (c % 2 == 1), c + 1, c)
    c = torch.where(y < 0, c + 128, c)
    return torch.where(y.isfinite(), c, torch.full_like(c, 127)).to(torch.uint8)


def exponent_for(top):
    """The smallest e with top <= 448 * 2^e, of 64-bit sizes, within -117 and 119."""
    torch = cu.torch_mod()
    m, k = torch.frexp(top)  # top = 2m 2^(k-1), and 448 = 1.75 2^8
    e = torch.where(m <= 0.875, k - 9, k - 8)
    return torch.where(top > 0, e, torch.full_like(e, -117)).clamp(-117, 119)


def where(D, values, device="cuda"):
    """The byte of (position, element) in a block, [16, D], by the header's formulas."""
    torch = cu.torch_mod()
    t, d = torch.arange(16, device=device)[:, None], torch.arange(D, device=device)[None]
    s, c, i = d // 64, d % 64 // 16, d % 16
    return 1024 * s + 256 * (t // 4) + 16 * i + 4 * c + t % 4 if values else 1024 * s + 64 * t + 16 * c + i


def rows_of(pool, values):
    """uint8 [..., page_len, D] by positions, of a pool as it is stored."""
    torch = cu.torch_mod()
    x = pool.view(torch.uint8)
    *lead, pl, D = x.shape
    return x.reshape(*lead, pl // 16, 16 * D)[..., where(D, values, x.device)].reshape(x.shape)


def stored(rows, values):
    """The inverse of rows_of, as float8_e4m3fn."""
    torch = cu.torch_mod()
    *lead, pl, D = rows.shape
    x = torch.empty(*lead, pl // 16, 16 * D, dtype=torch.uint8, device=rows.device)
    x[..., where(D, values, rows.device)] = rows.reshape(*lead, pl // 16, 16, D)
    return x.reshape(rows.shape).view(torch.float8_e4m3fn)


def exponents(scale):
    torch = cu.torch_mod()
    return scale.view(torch.uint8).int().clamp(10, 246) - 127


def numbers(codes):
    torch = cu.torch_mod()
    return torch.from_numpy(NUMBERS).to(codes.device)[codes.long()]


def decoded(pool, scale, values):
    """What a pool holds, in 64 bits, [..., page_len, D] by positions."""
    torch = cu.torch_mod()
    p = torch.exp2(exponents(scale).double()).repeat_interleave(16, -1)
    return numbers(rows_of(pool, values)) * p[..., None]


def runs(seqs, at, holds, max_seqs):
    """The tokens of a list by blocks: (first, last + 1); tokens without a place are left out."""
    i, n = 0, len(seqs)
    ok = [0 <= s < max_seqs and 0 <= p < holds for s, p in zip(seqs, at)]
    while i < n:
        j = i + 1
        while j < n and ok[i] and ok[j] and seqs[j] == seqs[i] and at[j] // 16 == at[i] // 16 and at[j] > at[j - 1]:
            j += 1
        if ok[i]:
            yield i, j
        i = j


class Written:
    """One layer's keys or values as the definition writes them: codes by positions (uint8
    [pages, G, page_len, D]) and exponents [pages, G, blocks]."""

    def __init__(self, pool, scale, values):
        self.codes, self.e = rows_of(pool, values).clone(), exponents(scale).clone()

    def append(self, x, seqs, at, table, max_seqs):
        """x: [n, G, D] in 64 bits."""
        torch = cu.torch_mod()
        P, G, pl, D = self.codes.shape
        for i, j in runs(seqs, at, table.shape[1] * pl, max_seqs):
            page, b = int(table[seqs[i], at[i] // pl]), at[i] % pl // 16
            if not 0 <= page < P:
                continue
            new = x[i:j]
            size = torch.where(new.isfinite(), new.abs(), torch.zeros_like(new))
            e = exponent_for(size.amax((0, 2)))
            block = self.codes[page, :, 16 * b:16 * b + 16]
            if at[i] % 16 == 0:
                block.zero_()
            else:
                old = self.e[page, :, b]
                e = torch.maximum(e, old)
                again = nearest(numbers(block) * torch.exp2((old - e).double())[:, None, None])
                nan = numbers(block).isnan()
                block.copy_(torch.where(nan, block, again))
            self.e[page, :, b] = e
            block[:, [p % 16 for p in at[i:j]]] = nearest(new / torch.exp2(e.double())[None, :, None]).transpose(0, 1)

    def same(self, pool, scale, values):
        """Equal in what the codes stand for (a zero has two signs, NaN several codes)."""
        a, b = numbers(rows_of(pool, values)), numbers(self.codes)
        return bool(((a == b) | (a.isnan() & b.isnan())).all()) and exponents(scale).equal(self.e)


def fill(cache, seed, spread=3):
    """N(0, 1)-like codes, scales around 2^-7 that differ from block to block."""
    torch = cu.torch_mod()
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    for pool, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        x = torch.randn(pool.shape, generator=g, device="cuda") * 100
        pool.copy_(x.clamp(-448, 448).to(torch.float8_e4m3fn))
        b = torch.randint(120 - spread, 121 + spread, scale.shape, generator=g, device="cuda")
        scale.view(torch.uint8).copy_(b.to(torch.uint8))
    return cache


def make(shape, lens, page_len=16, seed=0, layers=2, extra=0, spread=3):
    """A cache with scattered pages; everything that holds no token is NaN, blocks that hold none
    have scales out of range."""
    from paper_2608_27384_amd.flashvla import QuantCache
    torch = cu.torch_mod()
    dtype, H, G, D = shape
    need = [-(-n // page_len) for n in lens]
    total, width = sum(need) + 5, max(max(need), 1) + extra
    ids = np.random.default_rng(seed).permutation(total)
    table = np.full((len(lens), width), -1)
    refs, first = np.zeros(total), np.cumsum([0] + need)
    for b, n in enumerate(need):
        table[b, :n] = ids[first[b]:first[b + 1]]
    refs[ids[:first[-1]]] = 1
    cache = QuantCache.empty(layers, G, D, total, len(lens), width, page_len, cu.ttype(dtype))
    fill(cache, seed, spread)
    live = torch.zeros(total, page_len, dtype=torch.bool)
    for b, n in enumerate(lens):
        for j in range(need[b]):
            live[table[b, j], :min(page_len, n - j * page_len)] = True
    live = live.cuda()
    blocks = live.view(total, -1, 16).any(-1)
    for pool, scale, values in ((cache.k, cache.k_scale, False), (cache.v, cache.v_scale, True)):
        rows = rows_of(pool, values)
        rows[(~live)[None, :, None].expand(layers, total, G, page_len)] = 255
        pool.copy_(stored(rows, values))
        scale.view(torch.uint8)[(~blocks)[None, :, None].expand(scale.shape)] = 255
    cache.table.copy_(cu.ints(table))
    cache.length.copy_(cu.ints(lens))
    cache.refs.copy_(cu.ints(refs))
    return cache, cu.randn(dtype, seed + 3, len(lens), H, D), table


def context(cache, table, b, n, layer):
    """Keys and values of sequence b, [n, G, D] in 64 bits."""
    torch = cu.torch_mod()
    ids = [int(p) for p in table[b, :-(-n // cache.c.page_len)]]
    out = []
    for pool, scale, values in ((cache.k, cache.k_scale, False), (cache.v, cache.v_scale, True)):
        x = decoded(pool[layer:layer + 1].view(torch.uint8)[:, ids].view(torch.float8_e4m3fn),
                    scale[layer:layer + 1].view(torch.uint8)[:, ids].view(torch.float8_e8m0fnu), values)
        out.append(x[0].transpose(1, 2).reshape(-1, cache.c.n_kv_heads, cache.c.head_dim)[:n])
    return out


def attention(q, k, v, limits, dtype, scale=None):
    """cu.attention, with a bound that counts the sums of fp32 operands in three parts: three times
    as many terms (and the parts' sizes, which are 1 + 2^-7 + 2^-14 of a query at most) in a score's
    sum and in a result's.  Keys and values are exact, so no rounding of theirs counts."""
    out, size, soft = cu.attention(q, k, v, limits, scale)
    if dtype == "fp32" and len(k) and len(q):
        D = q.shape[-1]
        s = D ** -0.5 if scale is None else scale
        G = k.shape[1]
        S = max(float((q[:, h].double().abs() @ k[:, h * G // q.shape[1]].abs().t()).max()) for h in range(q.shape[1])) * s
        soft = soft + size * (2 * 2 * (D + 2) * 2.0 ** -24 * S + 2 * (len(k) + 64) * 2.0 ** -24) * (1 + 2.0 ** -6)
    return out, size, soft
