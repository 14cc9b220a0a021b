"""Plain 64-bit implementations of the cache operators and the inputs of their tests."""
import math

import numpy as np
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # relative error of one rounding to the type


def line_of(parent, i):
    """Chunk rows from row i up to the root, or None if the line leaves {-1, 0 .. i-1}."""
    rows = [i]
    while rows[-1] > 0:
        node = rows[-1] - 1
        p = int(parent[node])
        if p < -1 or p >= node:
            return None
        rows.append(p + 1)
    return rows


def random_tree(rng, nodes, k_cap, bad=0.0):
    par = np.full(k_cap, -1, np.int32)
    for i in range(nodes):
        par[i] = rng.integers(-1, i) if i and rng.random() < 0.8 else -1
        if i and rng.random() < 0.3:
            par[i] = i - 1
        if rng.random() < bad:
            par[i] = rng.choice([-2, i, i + 3, 1 << 30])
    return par


class Problem:
    """Chunks of a batch and a paged cache whose pages are in no order; what no request owns holds NaN."""

    def __init__(self, *, lens, rows, hq, hkv, d, page, dtype=torch.bfloat16, sel=None, k_cap=64, order="slots", tree=None, bad=0.0,
                 seed=0, device="cuda", extra_pages=2, sharp=2.0, uniform=False, pool_pages=None, table_extra=1):
        rng = np.random.default_rng(seed)
        g = torch.Generator(device=device).manual_seed(seed)
        self.B, self.hq, self.hkv, self.d, self.page, self.dtype, self.dev = len(lens), hq, hkv, d, page, dtype, device
        self.lens, self.rows, self.sel, self.k_cap = list(lens), list(rows), sel, k_cap
        self.n_new = [r if sel is None else min(max(0, min(s, k_cap)) + 1, r) for r, s in zip(rows, sel or rows)]
        self.total = sum(rows)
        self.k_uniform = rows[0] - 1 if uniform else 0
        self.off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int64)
        need = [max(1, -(-(n + m) // page)) for n, m in zip(self.lens, self.n_new)]
        width = max(need) + table_extra
        self.n_pages = pool_pages or sum(need) + extra_pages
        perm = rng.permutation(self.n_pages)[-sum(need):]
        self.table = np.full((self.B, width), -1, np.int32)
        for b, (o, n) in enumerate(zip(np.cumsum([0] + need), need)):
            self.table[b, :n] = perm[o:o + n]
        self.parent = None
        if tree is not None:
            self.parent = np.stack([random_tree(rng, max(0, m - 1), k_cap, bad) for m in self.n_new])
        randn = lambda *s: torch.randn(*s, generator=g, device=device).to(dtype)
        self.kd = [randn(n + m, hkv, d) for n, m in zip(self.lens, self.n_new)]
        self.vd = [randn(n + m, hkv, d) for n, m in zip(self.lens, self.n_new)]
        self.q = (randn(self.total, hq, d).float() * sharp).to(dtype)
        shape = (self.n_pages, page, hkv, d) if order == "slots" else (self.n_pages, hkv, page, d)
        self.k = torch.full(shape, float("nan"), dtype=dtype, device=device)
        self.v = torch.full(shape, float("nan"), dtype=dtype, device=device)
        if order == "heads":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)

    def places(self, b, lo, hi):
        t = np.arange(lo, hi)
        up = lambda x: torch.as_tensor(x, device=self.dev, dtype=torch.long)
        return up(self.table[b, t // self.page]), up(t % self.page)

    def fill(self, chunk=True):
        """The requests' tokens into their slots (chunk=False: only those before the chunk)."""
        for b in range(self.B):
            n = self.lens[b] + (self.n_new[b] if chunk else 0)
            if n:
                at = self.places(b, 0, n)
                self.k[at], self.v[at] = self.kd[b][:n], self.vd[b][:n]
        return self

    def device(self):
        up = lambda x, t: torch.as_tensor(np.asarray(x), dtype=t, device=self.dev)
        self.t_len, self.t_off = up(self.lens, torch.int32), up(self.off, torch.int64)
        self.t_sel = None if self.sel is None else up(self.sel, torch.int32)
        self.t_par = None if self.parent is None else up(self.parent, torch.int32)
        self.t_table = up(self.table, torch.int32)
        self.status = torch.full((self.B,), -5, dtype=torch.int32, device=self.dev)
        return self

    def context(self, **cfg):
        import paper_2606_01019_b200 as H
        ctx = H.Context(max_batch=max(self.B, 1), k_cap=self.k_cap, max_hist_len=16, max_rows=max(self.total, 1), max_vocab=8)
        ctx.hvd_set_attention(**{**dict(n_q_heads=self.hq, n_kv_heads=self.hkv, head_dim=self.d,
                                        dtype=H.BF16 if self.dtype == torch.bfloat16 else H.F16), **cfg})
        return ctx

    def cache(self):
        import paper_2606_01019_b200 as H
        return H.KvCache(self.k, self.v, self.t_table)


def sees(p, b, i):
    """The tokens that row i of request b sees, as a bool vector over lens + n_new."""
    n, m = p.lens[b], p.n_new[b]
    s = np.zeros(n + m, bool)
    if i >= m:
        return s
    if p.parent is None:
        s[:n + i + 1] = True
        return s
    rows = line_of(p.parent[b], i)
    if rows is not None:
        s[:n] = True
        s[n + np.array(rows)] = True
    return s


def attention(p, scale=None, kd=None, vd=None):
    """(out, lse, bound on |out|, largest sum of |products| of a score) in 64 bits: bound[row, head, e] = sum_j w_j |v_j|."""
    scale = 1.0 / math.sqrt(p.d) if scale is None else scale
    z = lambda *s: torch.zeros(*s, dtype=torch.float64, device=p.dev)
    out, size, lse, mass = z(p.total, p.hq, p.d), z(p.total, p.hq, p.d), z(p.total, p.hq) - math.inf, 0.0
    g = p.hq // p.hkv
    for b in range(p.B):
        if p.rows[b] == 0 or p.n_new[b] == 0:
            continue
        k = (kd or p.kd)[b].double().repeat_interleave(g, 1)   # [n, hq, d]
        v = (vd or p.vd)[b].double().repeat_interleave(g, 1)
        q = p.q[p.off[b]:p.off[b + 1]].double()
        m = torch.as_tensor(np.stack([sees(p, b, i) for i in range(p.rows[b])]), device=p.dev)
        x = torch.einsum("rhd,nhd->hrn", q, k) * scale
        mass = max(mass, float((torch.einsum("rhd,nhd->hrn", q.abs(), k.abs()) * scale).max()))
        x = x.masked_fill(~m[None], -math.inf)
        top = x.amax(-1, keepdim=True)
        w = torch.where(m[None], torch.exp(x - torch.where(torch.isinf(top), 0.0, top)), 0.0)
        l = w.sum(-1)
        some = (l > 0)[..., None]
        w = torch.where(some, w / torch.where(some, l[..., None], 1.0), 0.0)
        rows = slice(int(p.off[b]), int(p.off[b + 1]))
        out[rows] = torch.einsum("hrn,nhd->rhd", w, v)
        size[rows] = torch.einsum("hrn,nhd->rhd", w, v.abs())
        lse[rows] = torch.where(l > 0, top[..., 0] + torch.log(torch.where(l > 0, l, 1.0)), -math.inf).T
    return out, lse, size, mass


def check_attention(p, got, lse, want):
    """Each weight is rounded once to the type (u), the result once (u); a score is off by the rounding of a 32-bit
    accumulation of its products (2^-20 of their sum covers 128 products); exp2 and the division add 2^-18.  Weights
    below f16's normal numbers are off by at most 2^-25 of the largest, each."""
    out, wl, size, mass = want
    u = UNIT[p.dtype]
    score = 2.0 ** -20 * mass
    longest = max([n + m for n, m in zip(p.lens, p.n_new)] + [1])
    tail = longest * 2.0 ** -25 * 6.0 if p.dtype == torch.float16 else 0.0
    tol = (2 * u + 4 * score + 2.0 ** -18) * size + tail + (2.0 ** -25 if p.dtype == torch.float16 else 1e-37)
    bad = (got.double() - out).abs() > tol
    assert torch.isfinite(got.float()).all()
    assert not bad.any(), (int(bad.sum()), float(((got.double() - out).abs() / tol).max()))
    if lse is not None:
        none = torch.isinf(wl)
        assert torch.equal(torch.isinf(lse), none) and bool((lse[none] < 0).all())
        e = (lse.double() - wl)[~none].abs()
        assert e.numel() == 0 or bool((e <= 4 * score + 2.0 ** -18 + 2.0 ** -22 * wl[~none].abs()).all()), float(e.max())


def turned(x, pos, freq, mag, rot, pairs):
    """x [n, heads, d] rotated at positions pos [n], in 64 bits; also |x| + |y| of each element's pair."""
    x = x.double().clone()
    size = x.abs()
    a = pos.double()[:, None, None] * torch.as_tensor(freq, device=x.device)
    c, s = torch.cos(a) * mag, torch.sin(a) * mag
    i = torch.arange(rot // 2, device=x.device)
    first, second = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
    p, q = x[..., first].clone(), x[..., second].clone()
    x[..., first], x[..., second] = p * c - q * s, p * s + q * c
    size[..., first] = size[..., second] = (p.abs() + q.abs()) * mag
    return x, size
