"""Plain 64-bit forms of the observation context's operators, and the tolerances
that its GPU tests hold them to.

A rounding is off by at most half a step relative to the value: 2^-8 in bf16,
2^-24 in fp32.  With A = softmax(scores) |values|, an attention output may be off
by its own rounding (half a step of it), by that of every probability (bf16: half
a step of each, so 2^-8 A), by the scores (each product sum of dh terms off by at
most (dh + 2) 2^-24 of the sum of its terms' sizes S, which moves numerator and
denominator), by the hardware exponential and its argument (2^-22 and |argument|
2^-24, the argument at most 2 S log2 e), and by fp32 sums over n keys (n 2^-24)."""
import numpy as np

EPS = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def torch_mod():
    import torch
    return torch


def ttype(dtype):
    torch = torch_mod()
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def randn(dtype, seed, *shape, std=1.0):
    torch = torch_mod()
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(ttype(dtype))


def ints(a):
    torch = torch_mod()
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def attention(q, k, v, limits, scale=None):
    """q [n, H, D], k, v [m, G, D]; row i sees the keys below limits[i].  The result and the
    bound of an implementation's distance from it, without the storage type's roundings."""
    torch = torch_mod()
    n, H, D = q.shape
    m, G, _ = k.shape
    scale = D ** -0.5 if scale is None else scale
    out = torch.zeros(n, H, D, dtype=torch.float64, device=q.device)
    size = torch.zeros_like(out)
    if m == 0 or n == 0:
        return out, size, size
    see = torch.arange(m, device=q.device)[None] < torch.as_tensor(limits, device=q.device)[:, None]
    S = 0.0
    for h in range(H):
        kk, vv, qq = k[:, h * G // H].double(), v[:, h * G // H].double(), q[:, h].double()
        x = (qq @ kk.t() * scale).masked_fill(~see, -np.inf)
        p = torch.softmax(x, -1)
        p = torch.where(see.any(-1, keepdim=True), p, torch.zeros_like(p))
        p = torch.where(see, p, torch.zeros_like(p))
        out[:, h] = p @ vv
        size[:, h] = p @ vv.abs()
        S = max(S, float((qq.abs() @ kk.abs().t()).max()) * scale)
    soft = 2 * (D + 2) * 2.0 ** -24 * S + 2.0 ** -21 + 2 * 3 * S * 2.0 ** -24 + (m + 64) * 2.0 ** -24
    return out, size, size * soft


FEW, HALVES, TILES = range(3)


def prompt_form(dtype, n_q, n_k, prompts, heads, kv_heads, head_dim, causal):
    """The kernel that such a call of prompt attention takes (a C++ function of the library)."""
    import ctypes
    from paper_2608_27384_amd import flashvla as fvb
    torch_mod()  # its HIP runtime is the process's, if the library is not loaded before it
    f = getattr(fvb.lib(), "_ZN2fv11prompt_formERK14fv_prompt_args")
    f.restype, f.argtypes = ctypes.c_int, [ctypes.POINTER(fvb.FvPromptArgs)]
    a = fvb.FvPromptArgs(n_seqs=prompts, n_q=n_q, n_k=n_k, n_q_heads=heads, n_kv_heads=kv_heads,
                         head_dim=head_dim, dtype=fvb.FV_BF16 if dtype == "bf16" else fvb.FV_FP32,
                         causal=int(causal))
    return f(ctypes.byref(a))


def check_attention(got, ref, dtype):
    out, size, fp32 = ref
    tol = EPS[dtype] * out.abs() + fp32 * (1 + EPS[dtype]) + 1e-37
    if dtype == "bf16":
        tol = tol + EPS["bf16"] * size * (1 + EPS["bf16"])
    bad = ~((got.double() - out).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(),
                                 float((got.double() - out).abs().max()))


def check_attention_wide(got, ref, dtype):
    """The same where the probabilities of bf16 values are kept in two parts of bf16: of a
    probability in [1, 2) the first leaves less than 2^-7, which the second holds in steps of
    2^-15 at most, so half a step is 2^-16; as much of every other, by its exponent: 2^-16 A."""
    out, size, fp32 = ref
    tol = EPS[dtype] * out.abs() + fp32 * (1 + EPS[dtype]) + 1e-37
    if dtype == "bf16":
        tol = tol + 2.0 ** -16 * size * (1 + EPS["bf16"])
    bad = ~((got.double() - out).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(),
                                 float((got.double() - out).abs().max()))


def rotate(x, pos, sections, theta):
    """x [n, H, D] at positions pos [axes][n]: the 64-bit result, and its own size."""
    torch = torch_mod()
    D = x.shape[-1]
    axis = np.repeat(np.arange(len(sections)), sections)
    inv = float(np.float32(theta)) ** (-2.0 * np.arange(D // 2) / D)
    ang = torch.from_numpy(np.asarray(pos, np.float64)[axis].T * inv).to(x.device)[:, None]
    a, b = x[..., :D // 2].double(), x[..., D // 2:].double()
    c, s = torch.cos(ang), torch.sin(ang)
    size = (a.abs() * c.abs() + b.abs() * s.abs(), b.abs() * c.abs() + a.abs() * s.abs())
    whole = a.abs() + b.abs()
    return (torch.cat([a * c - b * s, b * c + a * s], -1), torch.cat(size, -1),
            torch.cat([whole, whole], -1))


def check_rotated(got, ref, dtype, angle_err=0.0):
    """Off by the output's rounding, three fp32 roundings of products and sum, and cosines and
    sines off by at most 2^-21 (the fraction of a turn in fp32, a library sine) + angle_err."""
    out, size, whole = ref
    tol = EPS[dtype] * out.abs() + 3 * 2.0 ** -24 * size + whole * (2.0 ** -21 + angle_err) + 1e-37
    tol = tol * (1 + EPS[dtype])
    assert bool(((got.double() - out).abs() <= tol).all()), float((got.double() - out).abs().max())


class Model:
    """The cache's bookkeeping in plain Python, one step at a time."""

    def __init__(self, n_pages, max_seqs, max_pages, page_len):
        self.pl, self.mp = page_len, max_pages
        self.table = np.full((max_seqs, max_pages), -1, np.int64)
        self.len = np.zeros(max_seqs, np.int64)
        self.refs = np.zeros(n_pages, np.int64)

    def pages(self, n):
        return -(-int(n) // self.pl)

    def _free(self):
        return [int(p) for p in np.nonzero(self.refs == 0)[0]]

    def _ok(self, s):
        return 0 <= s < len(self.len)

    def grow(self, seqs, add):
        if len(set(seqs)) != len(seqs):
            return 1
        need = 0
        for s, a in zip(seqs, add):
            if not self._ok(s) or a < 0 or self.len[s] + a > self.mp * self.pl:
                return 1
            n = int(self.len[s])
            if a > 0 and n % self.pl and self.refs[self.table[s, n // self.pl]] > 1:
                return 1
            need += self.pages(n + a) - self.pages(n)
        free = self._free()
        if need > len(free):
            return 2
        for s, a in zip(seqs, add):
            n = int(self.len[s])
            for j in range(self.pages(n), self.pages(n + a)):
                p = free.pop(0)
                self.table[s, j] = p
                self.refs[p] = 1
            self.len[s] = n + a
        return 0

    def fork(self, parents, children):
        """Status, and the page copies (source, destination, rows)."""
        if len(set(children)) != len(children) or not all(map(self._ok, list(parents) + list(children))):
            return 1, []
        if any(self.len[c] for c in children) or set(parents) & set(children):
            return 1, []
        free = self._free()
        if sum(1 for p in parents if self.len[p] % self.pl) > len(free):
            return 2, []
        copies = []
        for p, c in zip(parents, children):
            n = int(self.len[p])
            full, part = divmod(n, self.pl)
            self.table[c] = -1
            self.table[c, :full] = self.table[p, :full]
            for x in self.table[p, :full]:
                self.refs[x] += 1
            if part:
                d = free.pop(0)
                copies.append((int(self.table[p, full]), d, part))
                self.table[c, full] = d
                self.refs[d] = 1
            self.len[c] = n
        return 0, copies

    def free(self, seqs):
        if len(set(seqs)) != len(seqs) or not all(map(self._ok, seqs)):
            return 1
        for s in seqs:
            for x in self.table[s, :self.pages(self.len[s])]:
                self.refs[x] -= 1
            self.table[s] = -1
            self.len[s] = 0
        return 0

    def compact(self):
        """Pages in use, and the moves (source, destination)."""
        used = [int(p) for p in np.nonzero(self.refs)[0]]
        u = len(used)
        moves = list(zip([p for p in used if p >= u], [p for p in self._free() if p < u]))
        to = dict(moves)
        for s in range(len(self.len)):
            for j in range(self.pages(self.len[s])):
                self.table[s, j] = to.get(int(self.table[s, j]), self.table[s, j])
        for a, b in moves:
            self.refs[b], self.refs[a] = self.refs[a], 0
        return u, moves
