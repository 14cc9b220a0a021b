"""hvd_kv_commit against moving the rows one by one; everything else in the pools stays bit for bit."""
import numpy as np
import pytest
import torch

from tests import attn_reference as R

pytestmark = pytest.mark.gpu


class Commit:
    def __init__(self, B, nodes, layers, hkv=2, d=64, page=16, k_cap=64, order="slots", seed=0, dtype=torch.bfloat16, lens=None):
        rng = np.random.default_rng(seed)
        self.rng, self.layers, self.k_cap = rng, layers, k_cap
        lens = [int(x) for x in rng.integers(0, 200, B)] if lens is None else lens
        self.p = p = R.Problem(lens=lens, rows=[nodes + 1] * B, sel=[nodes] * B, hq=hkv, hkv=hkv, d=d, page=page, k_cap=k_cap, tree=True, seed=seed,
                               order=order, dtype=dtype).device()
        shape = (layers, p.n_pages, page, hkv, d) if order == "slots" else (layers, p.n_pages, hkv, page, d)
        bits = lambda: torch.randint(-32768, 32767, shape, device="cuda", dtype=torch.int16)   # any bit pattern, NaN among them
        self.k, self.v = bits().view(dtype), bits().view(dtype)
        if order == "heads":
            self.k, self.v = self.k.transpose(2, 3), self.v.transpose(2, 3)
        self.tok = rng.integers(0, 50, (B, k_cap)).astype(np.int32)      # equal siblings happen: the first child counts
        self.paths, self.com = [], np.full((B, k_cap + 1), -1, np.int32)
        for b in range(B):
            path, cur = [], -1
            while True:
                kids = [i for i in range(cur + 1, nodes) if p.parent[b, i] == cur]
                if not kids or rng.random() < 0.15:
                    break
                t = self.tok[b, rng.choice(kids)]
                cur = min(i for i in kids if self.tok[b, i] == t)
                self.com[b, len(path)] = t
                path.append(cur)
            self.com[b, len(path)] = 49 + b
            self.paths.append(path)
        self.accepted = np.array([len(x) for x in self.paths], np.int32)
        self.n_commit = self.accepted + 1

    def call(self, alias=False, chain=False, lens=None, n_commit=None):
        import paper_2606_01019_b200 as H
        p = self.p
        up = lambda x: torch.as_tensor(np.ascontiguousarray(x), device="cuda", dtype=torch.int32)
        ctx = p.context()
        cache = H.KvCache(self.k[0], self.v[0], p.t_table)
        ln = p.t_len.clone() if lens is None else up(lens)
        new = ln if alias else torch.full_like(ln, -9)
        tree = [None] * 5 if chain else [p.t_par, up(self.tok), p.t_sel, up(self.accepted), up(self.com)]
        ctx.hvd_kv_commit(p.B, cache, self.layers, self.k.stride(0), ln, *tree, up(self.n_commit if n_commit is None else n_commit), new)
        torch.cuda.synchronize()
        assert ctx.hvd_device_status() == 0
        ctx.close()
        return new.cpu().numpy()

    def expect(self, k, v, limit=None):
        p = self.p
        for b, path in enumerate(self.paths):
            for j, node in enumerate(path[:None if limit is None else limit[b]]):
                (pf, sf), (pt, st) = (p.places(b, p.lens[b] + 1 + x, p.lens[b] + 2 + x) for x in (node, j))
                for x in (k, v):
                    x[:, pt, st] = x[:, pf, sf].clone()
        return k, v


def same(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


@pytest.mark.parametrize("B,nodes,layers,kw", [(1, 1, 1, {}), (5, 32, 3, {}), (40, 64, 2, dict(order="heads", hkv=3, d=80)), (3, 64, 33, dict(page=8)),
                                               (9, 20, 4, dict(hkv=1, d=8, k_cap=20)), (300, 32, 2, dict(dtype=torch.float16)),
                                               (2, 63, 64, dict(hkv=8, d=128, page=32))])
@pytest.mark.parametrize("alias", [False, True])
def test_accepted_paths_become_consecutive(B, nodes, layers, kw, alias):
    c = Commit(B, nodes, layers, seed=B + nodes, **kw)
    k, v = c.expect(c.k.clone(), c.v.clone())
    new = c.call(alias)
    assert (new == np.array(c.p.lens) + c.n_commit).all()
    assert same(k, c.k) and same(v, c.v)
    assert B < 5 or max(len(x) for x in c.paths) >= 3


def test_a_chain_only_counts():
    c = Commit(6, 8, 2, seed=3)
    k, v = c.k.clone(), c.v.clone()
    assert (c.call(chain=True) == np.array(c.p.lens) + c.n_commit).all()
    assert same(k, c.k) and same(v, c.v)


def test_clamped_and_skipped_requests():
    """n_commit below accepted + 1 (a full slab), 0 or less (a skipped request), lengths that do not fit."""
    c = Commit(8, 40, 3, seed=4)
    c.paths[0] = c.paths[0][:0]
    n = c.n_commit.copy()
    n[0], n[1], n[2], n[3] = 0, -4, max(1, n[2] - 1), 1
    lens = np.array(c.p.lens)
    lens[4], lens[5] = -7, c.p.table.shape[1] * 16
    limit = [0, 0, n[2] - 1, 0, 0, 0] + [99] * 2
    k, v = c.expect(c.k.clone(), c.v.clone(), limit)
    new = c.call(lens=lens, n_commit=n)
    want = lens + np.where(n > 0, n, 0)
    want[4], want[5] = lens[4], lens[5]
    assert (new == want).all() and same(k, c.k) and same(v, c.v)


def test_a_path_that_ends_early_and_pages_outside_the_pool():
    c = Commit(6, 40, 2, seed=5, page=8, lens=[7, 15, 20, 31, 3, 0])
    c.accepted = c.accepted + 3                                     # says more than the tokens lead to
    c.n_commit = c.accepted + 1
    limit = [99] * 6
    b = max(range(6), key=lambda i: len(c.paths[i]))
    j = len(c.paths[b]) - 1
    c.p.table[b, (c.p.lens[b] + 1 + c.paths[b][j]) // 8] = -1
    c.p.device()
    pages = [{(c.p.lens[b] + 1 + x) // 8 for x in (n, i)} for i, n in enumerate(c.paths[b])]
    limit[b] = next(i for i, x in enumerate(pages) if any(c.p.table[b, y] < 0 for y in x))
    k, v = c.expect(c.k.clone(), c.v.clone(), limit)
    c.call()
    assert same(k, c.k) and same(v, c.v)


@pytest.mark.parametrize("alias", [False, True])
def test_the_verdict_of_every_request(alias):
    import paper_2606_01019_b200 as H
    c = Commit(8, 40, 3, seed=11, page=8, lens=[7, 15, 20, 31, 3, 0, 9, 50])
    longest = sorted(range(8), key=lambda i: -len(c.paths[i]))
    b, e, f = longest[:3]                                          # a page outside, a path that ends early, more nodes than the tree has
    assert len(c.paths[f]) >= 2
    want = np.zeros(8, np.int32)
    c.p.table[b, (c.p.lens[b] + 1 + c.paths[b][-1]) // 8] = c.p.n_pages
    want[b] = H.REQ_BAD_PAGE
    c.com[e, 1] = -77
    want[e] = H.REQ_BAD_PATH
    c.accepted[f], c.n_commit[f] = 41, 42
    want[f] = H.REQ_BAD_PATH
    rest = longest[3:]
    lens, n = np.array(c.p.lens), c.n_commit.copy()
    lens[rest[0]], lens[rest[1]] = -7, 8 * c.p.table.shape[1]
    want[rest[0]] = want[rest[1]] = H.REQ_BAD_LEN
    n[rest[2]], n[rest[3]] = 0, 1                                  # nothing to commit; the root alone
    width = 8 * c.p.table.shape[1]
    assert lens[f] + 42 <= width
    c.p.device()
    up = lambda x: torch.as_tensor(np.ascontiguousarray(x), device="cuda", dtype=torch.int32)
    ctx, ln = c.p.context(), up(lens)
    new, status = ln if alias else torch.full_like(ln, -9), torch.full_like(ln, -5)
    ctx.hvd_kv_commit(8, H.KvCache(c.k[0], c.v[0], c.p.t_table), 3, c.k.stride(0), ln, c.p.t_par, up(c.tok), c.p.t_sel, up(c.accepted), up(c.com), up(n),
                      new, status)
    assert status.tolist() == want.tolist()
    ok = lens + np.where((n > 0) & (want != H.REQ_BAD_LEN), n, 0)
    assert new.tolist() == ok.tolist()
    # chains
    ln, n = up([5, -1, width, 3]), up([2, 1, 1, 0])
    st = torch.full_like(ln, -5)
    ctx.hvd_kv_commit(4, H.KvCache(c.k[0], c.v[0], c.p.t_table), 3, c.k.stride(0), ln, None, None, None, None, None, n, torch.empty_like(ln), st)
    assert st.tolist() == [0, H.REQ_BAD_LEN, H.REQ_BAD_LEN, 0]
    ctx.close()


def test_refusals():
    import paper_2606_01019_b200 as H
    c = Commit(2, 4, 2)
    ctx, cache = c.p.context(), H.KvCache(c.k[0], c.v[0], c.p.t_table)
    n = c.p.t_len
    for text, a in (("n_layers", (2, cache, 0, 8, n, None, None, None, None, None, n, n)),
                    ("layer_stride", (2, cache, 2, 12, n, None, None, None, None, None, n, n)),
                    ("layer_stride", (2, cache, 2, 0, n, None, None, None, None, None, n, n)),
                    ("NULL", (2, cache, 1, 0, n, c.p.t_par, None, n, n, n, n, n)),
                    ("NULL", (2, cache, 1, 0, n, None, None, None, None, None, None, n)),
                    ("B outside", (3, cache, 1, 0, n, None, None, None, None, None, n, n))):
        with pytest.raises(H.HvdError, match=text):
            ctx.hvd_kv_commit(*a)
    ctx.close()
