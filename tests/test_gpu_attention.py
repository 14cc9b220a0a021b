"""hvd_attn_paged against softmax attention in 64 bits."""
import numpy as np
import pytest
import torch

from tests import attn_reference as R

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def run(p, ctx=None, lse=True, q=None, out=None, row_off=True, cache=None, **cfg):
    p.device()
    own = ctx is None
    ctx = ctx or p.context(**cfg)
    q = p.q if q is None else q
    out = torch.full((p.total, p.hq, p.d), float("nan"), dtype=p.dtype, device="cuda") if out is None else out
    ls = torch.full((p.total, p.hq), float("nan"), device="cuda") if lse else None
    ctx.hvd_attn_paged(p.B, cache or p.cache(), p.t_len, p.t_off if row_off else None, p.k_uniform, p.total, p.t_sel, p.t_par, q,
                       out, ls, p.status)
    torch.cuda.synchronize()
    assert ctx.hvd_device_status() == 0
    if own:
        ctx.close()
    return out, ls


def check(p, scale=None, **kw):
    p.fill()
    out, lse = run(p, **({} if scale is None else dict(softmax_scale=scale)), **kw)
    R.check_attention(p, out, lse, R.attention(p, scale))
    assert (p.status == 0).all()
    return out, lse


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [8, 16, 64, 72, 80, 96, 120, 128])
def test_head_dims(d, dtype):
    check(R.Problem(lens=[0, 1, 127, 300], rows=[3, 1, 9, 5], hq=8, hkv=2, d=d, page=16, dtype=dtype, seed=d))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (3, 1), (10, 2), (12, 4), (7, 1), (32, 4), (128, 1), (33, 3)])
def test_head_groups(hq, hkv):
    check(R.Problem(lens=[5, 140, 260], rows=[1, 17, 40], hq=hq, hkv=hkv, d=64, page=32, seed=hq))


@pytest.mark.parametrize("page", [8, 16, 24, 40, 48, 64, 128, 136, 256, 1024])
@pytest.mark.parametrize("order", ["slots", "heads"])
def test_page_sizes(page, order):
    check(R.Problem(lens=[1, 7, 129, 383, 700], rows=[2, 9, 1, 17, 4], hq=4, hkv=2, d=128, page=page, order=order, seed=page))


@pytest.mark.parametrize("n", [0, 1, 2, 7, 8, 31, 62, 63, 64, 126, 127, 128, 129, 254, 255, 256, 257, 383, 511, 1000, 2049])
def test_lengths_around_the_tile(n):
    check(R.Problem(lens=[n, n + 1], rows=[1, 2], hq=4, hkv=1, d=128, page=16, seed=n))


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 385, 600])
@pytest.mark.parametrize("hq", [1, 4])
def test_chunk_lengths(rows, hq):
    """One to several tiles of query rows; the causal edge inside and on the border of key tiles."""
    check(R.Problem(lens=[0, 100], rows=[rows, rows], hq=hq, hkv=1, d=64, page=16, seed=rows))


def test_rows_from_k_uniform_and_ragged_selection():
    p = R.Problem(lens=[40, 0, 333, 129], rows=[17] * 4, sel=[16, 0, 5, 99], k_cap=16, hq=8, hkv=2, d=128, page=16, uniform=True)
    out, lse = check(p, row_off=False)
    for b, m in enumerate(p.n_new):                            # rows that are no new token
        r = slice(int(p.off[b]) + m, int(p.off[b + 1]))
        assert (out[r] == 0).all() and torch.isinf(lse[r]).all()


@pytest.mark.parametrize("B", [383, 384, 385, 900, 2100])
def test_batches_of_more_requests_than_a_cta_has_threads(B):
    rng = np.random.default_rng(B)
    check(R.Problem(lens=[int(x) for x in rng.integers(0, 200, B)], rows=[int(x) for x in rng.integers(0, 4, B)], hq=6, hkv=3, d=32, page=16, seed=B))


def test_many_rows_that_are_no_new_token():
    """Short drafts in wide blocks of rows, as a ragged batch has them: the other rows come out as zeros."""
    rng = np.random.default_rng(4)
    B = 200
    p = R.Problem(lens=[int(x) for x in rng.integers(0, 90, B)], rows=[33] * B, sel=[int(x) for x in rng.integers(-1, 4, B)], hq=5, hkv=1, d=80,
                  page=16, seed=4)
    out, lse = check(p)
    rest = np.concatenate([np.arange(p.off[b] + p.n_new[b], p.off[b + 1]) for b in range(B)])
    assert (out[rest] == 0).all() and torch.isinf(lse[rest]).all()


def test_empty_requests_and_an_empty_batch():
    check(R.Problem(lens=[10, 0, 50, 3], rows=[0, 0, 4, 0], hq=4, hkv=2, d=64, page=16))
    p = R.Problem(lens=[10, 0], rows=[0, 0], hq=4, hkv=2, d=64, page=16)
    check(p)


@pytest.mark.parametrize("nodes,hq,hkv,dtype", [(1, 4, 1, BF), (32, 8, 2, BF), (64, 16, 2, HF), (64, 4, 4, BF), (33, 24, 3, BF)])
def test_trees(nodes, hq, hkv, dtype):
    rng = np.random.default_rng(nodes)
    B = 6
    sel = [nodes, max(0, nodes - 1), 0, nodes // 2, nodes, nodes]
    check(R.Problem(lens=[0, 1, 200, 255, 127, int(rng.integers(0, 900))], rows=[nodes + 1] * B, sel=sel, hq=hq, hkv=hkv, d=64,
                    page=16, dtype=dtype, tree=True, seed=nodes))


def test_unreachable_nodes_see_nothing():
    p = R.Problem(lens=[100, 30, 0], rows=[33] * 3, sel=[32] * 3, hq=4, hkv=1, d=64, page=16, tree=True, bad=0.2, seed=5)
    out, lse = check(p)
    lost = [int(p.off[b]) + i for b in range(3) for i in range(33) if R.line_of(p.parent[b], i) is None]
    assert len(lost) > 5 and (out[lost] == 0).all() and torch.isinf(lse[lost]).all()


def test_a_chain_as_a_tree_gives_the_chain():
    kw = dict(lens=[77, 128, 0], rows=[20, 9, 33], sel=[19, 8, 32], hq=8, hkv=2, d=128, page=16, seed=3)
    a, b = R.Problem(**kw), R.Problem(**kw)
    b.parent = np.tile(np.arange(-1, 63, dtype=np.int32), (3, 1))
    for x, y in zip(check(a), check(b)):
        assert torch.equal(x, y)


def test_strided_rows():
    """q a slice of a fused projection, out inside a wider array."""
    p = R.Problem(lens=[50, 300], rows=[9, 17], hq=8, hkv=2, d=64, page=16, seed=9)
    wide = torch.full((p.total, p.hq + 4, 80), float("nan"), dtype=BF, device="cuda")
    wide[:, 2:10, 8:72] = p.q
    room = torch.full((p.total, 3, p.hq, 72), 7.0, dtype=BF, device="cuda")
    out = room[:, 1, :, :64]
    check(p, q=wide[:, 2:10, 8:72], out=out)
    assert (room[:, 0] == 7).all() and (room[:, 2] == 7).all() and (room[:, 1, :, 64:] == 7).all()


@pytest.mark.parametrize("scale", [0.01, 0.5, 3.0])
def test_softmax_scale(scale):
    check(R.Problem(lens=[400, 90], rows=[5, 40], hq=4, hkv=2, d=64, page=16, seed=1, sharp=1.0), scale=scale)


def test_maxima_that_climb_and_fall():
    """Scores that rise by hundreds along the keys, stay far below zero, or are all equal."""
    p = R.Problem(lens=[1500, 1500, 1500, 600], rows=[9, 9, 9, 70], hq=4, hkv=1, d=64, page=16, seed=2)
    one = torch.ones(64, device="cuda")
    p.q = torch.ones_like(p.q)
    for b, f in enumerate([lambda n: torch.linspace(-60, 60, n), lambda n: torch.linspace(60, -60, n), lambda n: torch.full((n,), -90.0),
                           lambda n: torch.linspace(-20, 20, n)]):
        p.kd[b] = (f(p.kd[b].shape[0]).cuda()[:, None, None] * one / 8).to(BF).expand_as(p.kd[b]).contiguous()
    check(p)


@pytest.mark.parametrize("hq,d,dtype", [(1, 128, BF), (4, 128, BF), (16, 64, HF)])
def test_queries_that_are_nan_stay_in_their_own_request(hq, d, dtype):
    """Requests of one row are worked on where requests of whole row tiles were before them: what those left in the part of the
    query tile that one row does not use reaches no result, not by one bit."""
    rng = np.random.default_rng(hq)
    B = 600
    rows = [int(rng.integers(64, 300)) // hq + 1 if b % 2 == 0 else int(rng.integers(1, 4)) for b in range(B)]
    p = R.Problem(lens=[int(x) for x in rng.integers(0, 400, B)], rows=rows, hq=hq, hkv=1, d=d, page=16, dtype=dtype, seed=hq).fill()
    out, lse = run(p)
    want = R.attention(p)
    R.check_attention(p, out, lse, want)
    short = np.concatenate([np.arange(p.off[b], p.off[b + 1]) for b in range(1, B, 2)])
    wide = np.concatenate([np.arange(p.off[b], p.off[b + 1]) for b in range(0, B, 2)])
    q = p.q.clone()
    q[wide] = torch.tensor([float("nan"), float("inf"), 60000.0], dtype=dtype, device=q.device)[torch.arange(len(wide), device=q.device) % 3][:, None, None]
    got, got_lse = run(p, q=q)
    assert torch.equal(got[short], out[short]) and torch.equal(got_lse[short], lse[short])


def test_slots_behind_the_chunk_may_hold_anything():
    for fill in (float("nan"), float("inf"), -float("inf"), 3.0e38):
        p = R.Problem(lens=[100, 37, 127, 0], rows=[3, 1, 1, 1], hq=4, hkv=2, d=128, page=64, seed=4)
        p.k.fill_(fill)
        p.v.fill_(fill)
        check(p)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("hq", [2, 32])
def test_infinite_tokens_stay_with_the_rows_that_see_them(hq, tree, dtype):
    """NaN and infinities in k or v of some of the chunk's tokens: rows that do not see them come out as if they were zeros; rows
    that do get the infinity or NaN in its elements (v) or NaN throughout (k)."""
    kw = dict(lens=[100, 60, 0, 700], rows=[20, 33, 40, 65], sel=[19, 32, 39, 64], hq=hq, hkv=2, d=80, page=16, dtype=dtype,
              tree=True if tree else None, bad=0.1, seed=3)
    clean, p = R.Problem(**kw), R.Problem(**kw)
    bad_v = {(0, 3): [5, 70], (0, 19): [0], (1, 1): [79], (1, 20): [8, 9], (2, 0): [1], (3, 40): [33], (3, 64): [2]}
    bad_k = {(0, 7), (3, 50)}
    for n, ((b, i), cols) in enumerate(bad_v.items()):
        p.vd[b][p.lens[b] + i, :, cols] = [float("inf"), float("nan"), -float("inf")][n % 3]
        clean.vd[b][p.lens[b] + i, :, cols] = 0
    for b, i in bad_k:
        p.kd[b][p.lens[b] + i] = float("nan")
        clean.kd[b][p.lens[b] + i] = 0
    out, lse = run(p.fill())
    want = R.attention(clean)
    hit = torch.zeros(p.total, p.d, dtype=torch.bool, device="cuda")
    lost = torch.zeros(p.total, dtype=torch.bool, device="cuda")
    for b in range(p.B):
        for i in range(p.rows[b]):
            s = R.sees(p, b, i)
            for (bb, j), cols in bad_v.items():
                if bb == b and s[p.lens[b] + j]:
                    hit[p.off[b] + i, cols] = True
            lost[p.off[b] + i] = any(bb == b and s[p.lens[b] + j] for bb, j in bad_k)
    assert hit.any() and lost.any() and not lost.all()
    fine = ~hit & ~lost[:, None]
    assert not torch.isfinite(out.float())[(hit & ~lost[:, None])[:, None].expand_as(out)].any()
    mask = fine[:, None].expand_as(out)
    got = torch.where(mask, out.float(), 0.0)
    ls = torch.where(lost[:, None], 0.0, lse)
    R.check_attention(clean, got, ls, (torch.where(mask, want[0], 0.0), torch.where(lost[:, None], 0.0, want[1]), *want[2:]))


def test_values_of_the_prompt_that_are_infinite_leave_empty_rows_empty():
    p = R.Problem(lens=[300, 40], rows=[9, 9], sel=[8, 8], hq=4, hkv=2, d=64, page=16, tree=True, seed=2)
    p.parent[:, 4] = 60                                        # unreachable: sees nothing
    for v in p.vd:
        v[5] = float("nan")
    out, lse = run(p.fill())
    rows = [int(p.off[b]) + i for b in range(2) for i in range(9) if R.line_of(p.parent[b], i) is None]
    assert (out[rows] == 0).all() and torch.isinf(lse[rows]).all() and len(rows) >= 2


def check_but(lost, p, out, lse, want):
    """The rows and heads of `lost` [total, hq] are NaN throughout, the others as in 64 bits."""
    assert lost.any()
    assert torch.isnan(out[lost]).all() and torch.isnan(lse[lost]).all()
    keep = ~lost
    rest = lambda x: torch.where(keep[..., None], x, 0.0)
    R.check_attention(p, rest(out.float()), torch.where(keep, lse, 0.0),
                      (rest(want[0]), torch.where(keep, want[1], 0.0), rest(want[2]), want[3]))


def rows_that_see(p, b, t):
    """[total] rows of the batch that see token t of request b."""
    s = torch.zeros(p.total, dtype=torch.bool, device="cuda")
    for i in range(p.rows[b]):
        s[p.off[b] + i] = bool(R.sees(p, b, i)[t])
    return s


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 2), (32, 1)])
def test_a_nan_key_makes_the_rows_that_see_it_nan(hq, hkv, tree, dtype):
    """Keys of the prompt and of the chunk, the only key of a row among them; items of one piece and of many."""
    kw = dict(lens=[0, 100, 0, 9000, 60], rows=[1, 20, 33, 9, 30], sel=[0, 19, 32, 8, 29], hq=hq, hkv=hkv, d=64, page=16, dtype=dtype,
              tree=True if tree else None, bad=0.1, seed=21)
    clean, p = R.Problem(**kw), R.Problem(**kw)
    lost = torch.zeros(p.total, dtype=torch.bool, device="cuda")
    for b, t in ((0, 0), (1, 100 + 5), (1, 100 + 9), (2, 3), (3, 4003), (4, 60 + 8)):
        p.kd[b][t] = float("nan")
        clean.kd[b][t] = 0
        lost |= rows_that_see(p, b, t)
    assert not lost.all()
    out, lse = run(p.fill())
    check_but(lost[:, None].expand(p.total, hq), p, out, lse, R.attention(clean))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("hq,hkv,rows", [(1, 1, 1), (8, 2, 9), (8, 2, 40), (32, 1, 9)])
def test_a_nan_query_makes_its_own_row_nan(hq, hkv, rows, dtype):
    kw = dict(lens=[0, 37, 700, 20000], rows=[rows] * 4, hq=hq, hkv=hkv, d=64, page=16, dtype=dtype, seed=22)
    clean, p = R.Problem(**kw), R.Problem(**kw)
    lost = torch.rand(p.total, hq, generator=torch.Generator("cuda").manual_seed(1), device="cuda") < 0.3
    lost[0, 0], lost[-1, -1] = True, True
    p.q[lost] = float("nan")
    clean.q[lost] = 0
    out, lse = run(p.fill())
    check_but(lost, p, out, lse, R.attention(clean))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("n,rows", [(0, 1), (30, 5), (200, 70), (9000, 3)])
def test_scores_that_are_all_minus_infinity(n, rows, dtype):
    """A row whose scores are all -infinity sees keys all the same: by the formula 0 / 0 in out, log 0 in lse.  Unreachable rows beside it
    see nothing and come out as zeros."""
    nodes = rows - 1
    p = R.Problem(lens=[n, 50], rows=[rows, rows], sel=[min(nodes, 64), nodes], hq=4, hkv=1, d=64, page=16, dtype=dtype, tree=True, bad=0.3, seed=23)
    q, k = p.q, p.kd[0]
    q[..., 0] = 1.0
    k[:, :, 0] = -float("inf")
    out, lse = run(p.fill())
    seen = torch.tensor([bool(R.sees(p, 0, i).any()) for i in range(rows)], device="cuda")
    first, first_lse = out[:rows], lse[:rows]
    assert torch.isnan(first[seen]).all() and (first[~seen] == 0).all()
    assert (first_lse == -float("inf")).all()
    want = R.attention(p)
    there = torch.arange(p.total, device="cuda")[:, None] >= rows
    mass = float(torch.einsum("rhd,nd->hrn", q[rows:].double().abs(), p.kd[1][:, 0].double().abs()).max()) / 8.0
    R.check_attention(p, torch.where(there[..., None], out.float(), 0.0), torch.where(there, lse, 0.0),
                      (torch.where(there[..., None], want[0], 0.0), torch.where(there, want[1], 0.0), torch.where(there[..., None], want[2], 0.0), mass))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,hq", [(1, 4), (40, 8)])
@pytest.mark.parametrize("n", [200, 5000])
def test_a_nan_key_shows_at_every_column(n, rows, hq, dtype):
    """Request c has its NaN key in column c of a tile."""
    p = R.Problem(lens=[n] * 64, rows=[rows] * 64, hq=hq, hkv=1, d=64, page=16, dtype=dtype, seed=24)
    for c in range(64):
        p.kd[c][64 + c] = float("nan")
    out, lse = run(p.fill())
    assert torch.isnan(out).all() and torch.isnan(lse).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,hq", [(1, 4), (40, 8)])
@pytest.mark.parametrize("n", [200, 5000])
def test_an_infinite_score_shows_at_every_column(n, rows, hq, dtype):
    """Request c has its infinite key in column c of a tile.  Heads with a positive element make a score of +infinity of it (inf / inf
    in out), the others one of -infinity: a weight of zero, like that of a score far below the rest."""
    kw = dict(lens=[n] * 64, rows=[rows] * 64, hq=hq, hkv=1, d=64, page=16, dtype=dtype, seed=24)
    clean, p = R.Problem(**kw), R.Problem(**kw)
    up = torch.arange(hq, device="cuda") % 2 == 0
    p.q[..., 0] = torch.where(up, 1.0, -1.0).to(dtype)
    clean.q[..., 0] = p.q[..., 0]
    for c in range(64):
        p.kd[c][64 + c], clean.kd[c][64 + c] = 0.0, 0.0
        p.kd[c][64 + c, :, 0], clean.kd[c][64 + c, :, 0] = float("inf"), 2000.0   # 250 below
    out, lse = run(p.fill())
    check_but(up[None].expand(p.total, hq), p, out, lse, R.attention(clean))


def test_a_non_finite_value_costs_its_own_item_only():
    """2048 requests of one wide item each, some 14 to an SM.  One value of one chunk is NaN: whether that item is the first or the last
    of its SM's makes no difference to the call's time (its own rows pay, 13 others do not: a factor of 14 otherwise, so 4 tells them apart)."""
    B, rows = 2048, 64
    p = R.Problem(lens=[64] * B, rows=[rows] * B, hq=4, hkv=1, d=64, page=64, seed=25).fill().device()
    ctx, cache, out = p.context(), p.cache(), torch.empty_like(p.q)

    def took(b):
        at = p.places(b, 64 + rows - 1, 64 + rows)
        was = p.v[at].clone()
        p.v[at] = torch.where(torch.arange(64, device="cuda") == 5, float("nan"), was.float()).to(BF)
        times = []
        for _ in range(6):
            s, e = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            s.record()
            ctx.hvd_attn_paged(B, cache, p.t_len, p.t_off, 0, p.total, None, None, p.q, out)
            e.record()
            e.synchronize()
            times.append(s.elapsed_time(e))
        assert torch.isnan(out[b * rows + rows - 1, :, 5]).all() and torch.isfinite(out[b * rows + rows - 2]).all()
        p.v[at] = was
        return min(times[2:])
    first, last = took(0), took(B - 1)
    assert first < 4 * last, (first, last)
    ctx.close()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("n", [32767, 131071])
def test_the_sum_of_many_small_weights(n, dtype):
    """One key stands 17.5 above all the others, which together add n e^-17.5 to the sum of weights: to 32 bits a tile of them is a few units
    in the last place of the whole.  Rounding of the sum below 2^-18 of it, of exponent and logarithm below 2^-22 of 20; 160 requests
    of two heads on the same pages, so that most are worked on in one piece."""
    import paper_2606_01019_b200 as H
    B, page = 160, 64
    pages = -(-(n + 1) // page)
    k = torch.zeros(pages, page, 2, 64, dtype=dtype, device="cuda")
    k[0, 0, :, 0] = 14.0
    q = torch.zeros(B, 2, 64, dtype=dtype, device="cuda")
    q[..., 0] = 10.0
    table = torch.arange(pages, dtype=torch.int32, device="cuda").expand(B, pages).contiguous()
    ctx = H.Context(max_batch=B, k_cap=1, max_hist_len=16, max_rows=B, max_vocab=8)
    ctx.hvd_set_attention(n_q_heads=2, n_kv_heads=2, head_dim=64, dtype=H.BF16 if dtype is BF else H.F16)
    out, lse = torch.empty_like(q), torch.empty(B, 2, device="cuda")
    ctx.hvd_attn_paged(B, H.KvCache(k, k.clone(), table), torch.full((B,), n, dtype=torch.int32, device="cuda"), None, 0, B, None, None, q, out, lse)
    e = (lse.double() - (17.5 + np.log1p(n * np.exp(-17.5)))).abs()
    assert bool((e <= 2.0 ** -17 + 2.0 ** -22 * 20).all()), float(e.max())
    assert ctx.hvd_device_status() == 0
    ctx.close()


@pytest.mark.parametrize("n", [2000, 32767, 131071])
@pytest.mark.parametrize("rows", [1, 9])
def test_many_small_weights_behind_a_large_one_f16(n, rows):
    """One key stands 17.5 above all the others, whose values are 1 where its own is 0.  A weight that small is below half of f16's smallest
    number; held against a maximum of 2^7 it is not lost.  Each is off by 2^-25 of 2^-7 at most, the result is rounded once; 320 requests
    on the same pages, so that most are worked on in one piece."""
    import paper_2606_01019_b200 as H
    B, page, end = 320, 64, n + rows
    pages = -(-end // page)
    k, v = torch.zeros(pages, page, 1, 64, dtype=HF, device="cuda"), torch.ones(pages, page, 1, 64, dtype=HF, device="cuda")
    k[0, 0, 0, 0], v[0, 0] = 14.0, 0.0
    q = torch.zeros(B * rows, 16, 64, dtype=HF, device="cuda")
    q[..., 0] = 10.0
    table = torch.arange(pages, dtype=torch.int32, device="cuda").expand(B, pages).contiguous()
    ctx = H.Context(max_batch=B, k_cap=16, max_hist_len=16, max_rows=B * rows, max_vocab=8)
    ctx.hvd_set_attention(n_q_heads=16, n_kv_heads=1, head_dim=64, dtype=H.F16)
    out, lse = torch.empty_like(q), torch.empty(B * rows, 16, device="cuda")
    ctx.hvd_attn_paged(B, H.KvCache(k, v, table), torch.full((B,), n, dtype=torch.int32, device="cuda"), None, rows - 1, B * rows, None, None, q, out, lse)
    seen = n + 1 + np.arange(rows)                       # keys of each row
    tail = (seen - 1) * np.exp(-17.5)
    want = torch.as_tensor(np.tile(tail / (1 + tail), B), device="cuda")[:, None, None]
    tol = (2 * R.UNIT[HF] + 2.0 ** -18) * want + n * 2.0 ** -32 + 2.0 ** -25
    e = (out.double() - want).abs()
    assert bool((e <= tol).all()), float((e / tol).max())
    want_lse = torch.as_tensor(np.tile(17.5 + np.log1p(tail), B), device="cuda")[:, None]
    assert bool(((lse.double() - want_lse).abs() <= 2.0 ** -17 + 2.0 ** -22 * 20).all())
    assert ctx.hvd_device_status() == 0
    ctx.close()


def test_unusable_requests_are_skipped():
    p = R.Problem(lens=[20, 20, 20, 20, 20], rows=[4, 5, 6, 3, 2], sel=[3, 4, 5, 2, 1], hq=4, hkv=2, d=64, page=16, seed=6).fill()
    want = R.attention(p)
    p.device()
    ctx = p.context()
    lens = p.t_len.clone()
    lens[1], lens[3] = -1, p.table.shape[1] * 16 - 2           # one row too many for the table
    out, lse = torch.full_like(p.q, 5.0), torch.full((p.total, p.hq), 5.0, device="cuda")
    ctx.hvd_attn_paged(p.B, p.cache(), lens, p.t_off, 0, p.total, p.t_sel, None, p.q, out, lse, p.status)
    assert p.status.tolist() == [0, 2, 0, 2, 0]
    for b in (1, 3):
        r = slice(int(p.off[b]), int(p.off[b + 1]))
        assert (out[r] == 0).all() and torch.isinf(lse[r]).all()
        want[0][r], want[1][r], want[2][r] = 0, -np.inf, 0
    R.check_attention(p, out, lse, want)
    # rows outside the arrays, rows that run backwards
    off = p.t_off.clone()
    off[2], off[5] = 1000, -7
    ctx.hvd_attn_paged(p.B, p.cache(), p.t_len, off, 0, p.total, p.t_sel, None, p.q, out, lse, p.status)
    assert p.status.tolist() == [0, 2, 2, 0, 2]
    assert ctx.hvd_device_status() == 0
    ctx.close()


def test_page_entries_outside_the_pool_stand_for_zeros():
    p = R.Problem(lens=[100, 60], rows=[3, 2], hq=4, hkv=2, d=64, page=16, seed=7).fill()
    kd, vd = [x.clone() for x in p.kd], [x.clone() for x in p.vd]
    for b, j, v in ((0, 2, -1), (0, 4, p.n_pages), (1, 0, 2 ** 31 - 1)):
        p.table[b, j] = v
        kd[b][16 * j:16 * j + 16] = 0
        vd[b][16 * j:16 * j + 16] = 0
    out, lse = run(p)
    R.check_attention(p, out, lse, R.attention(p, kd=kd, vd=vd))


def test_a_cache_that_ends_in_the_last_tile_below_2_to_31():
    """Every page of the table but the last is the same one; keys of zeros, values of ones.  What lies behind the last token is NaN."""
    import paper_2606_01019_b200 as H
    page, width = 65528, 32772
    end = page * width - 4
    k, v = torch.zeros(2, page, 1, 8, dtype=BF, device="cuda"), torch.ones(2, page, 1, 8, dtype=BF, device="cuda")
    k[1, -4:], v[1, -4:] = float("nan"), float("nan")
    table = torch.zeros(1, width, dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    ctx = H.Context(max_batch=1, k_cap=1, max_hist_len=16, max_rows=1, max_vocab=8)
    ctx.hvd_set_attention(n_q_heads=1, n_kv_heads=1, head_dim=8)
    q, out, lse = torch.ones(1, 1, 8, dtype=BF, device="cuda"), torch.empty(1, 1, 8, dtype=BF, device="cuda"), torch.empty(1, 1, device="cuda")
    ctx.hvd_attn_paged(1, H.KvCache(k, v, table), torch.tensor([end - 1], dtype=torch.int32, device="cuda"), None, 0, 1, None, None, q, out, lse)
    assert (out == 1).all() and abs(float(lse) - np.log(end)) < 1e-5
    assert ctx.hvd_device_status() == 0
    ctx.close()


def test_long_ragged_batch_split_over_the_sms():
    """Contexts from one token to 40 000: most are cut into pieces that are joined again."""
    rng = np.random.default_rng(8)
    lens = [int(x) for x in np.exp(rng.uniform(0, np.log(20000), 24))] + [40001]
    check(R.Problem(lens=lens, rows=[int(x) for x in rng.integers(1, 18, 25)], hq=8, hkv=2, d=64, page=16, seed=8))


@pytest.mark.parametrize("lens,rows,hq,hkv,d", [([30000], [1], 32, 8, 128), ([9001], [65], 16, 2, 128), ([50], [700], 16, 2, 128),
                                                ([12345, 3], [64, 300], 8, 1, 128)])
def test_few_requests(lens, rows, hq, hkv, d):
    check(R.Problem(lens=lens, rows=rows, hq=hq, hkv=hkv, d=d, page=32, seed=11))


def test_results_do_not_depend_on_the_run():
    p = R.Problem(lens=[5000, 130, 2222], rows=[9, 17, 1], hq=8, hkv=2, d=128, page=16, seed=12).fill()
    p.device()
    ctx = p.context()
    first = None
    for _ in range(4):
        out, lse = run(p, ctx=ctx)
        first = first or (out, lse)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    ctx.close()


def test_another_stream_and_a_graph():
    p = R.Problem(lens=[700, 1300], rows=[9, 9], hq=8, hkv=2, d=128, page=16, seed=13).fill()
    want = R.attention(p)
    p.device()
    ctx, cache, out, lse = p.context(), p.cache(), torch.zeros_like(p.q), torch.zeros(p.total, p.hq, device="cuda")
    call = lambda: ctx.hvd_attn_paged(p.B, cache, p.t_len, p.t_off, 0, p.total, None, None, p.q, out, lse, p.status)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    s.synchronize()
    R.check_attention(p, out, lse, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    out.zero_(), lse.zero_()
    g.replay(), g.replay()
    torch.cuda.synchronize()
    R.check_attention(p, out, lse, want)
    del g
    ctx.close()


def test_a_graph_outlives_another_geometry():
    """A graph captured with heads of 64 runs after the context has been set to heads of 128 and used with them."""
    p = R.Problem(lens=[3000, 1300], rows=[9, 9], hq=8, hkv=2, d=64, page=16, seed=26).fill().device()
    wide = R.Problem(lens=[3000, 1300], rows=[9, 9], hq=8, hkv=2, d=128, page=16, seed=27).fill()
    ctx, cache, out, lse = p.context(), p.cache(), torch.zeros_like(p.q), torch.zeros(p.total, p.hq, device="cuda")
    call = lambda: ctx.hvd_attn_paged(p.B, cache, p.t_len, p.t_off, 0, p.total, None, None, p.q, out, lse)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    ctx.hvd_set_attention(n_q_heads=8, n_kv_heads=2, head_dim=128)
    R.check_attention(wide, *run(wide, ctx=ctx), R.attention(wide))
    filler = torch.full((48 << 20,), 0x7f, dtype=torch.uint8, device="cuda")
    out.zero_(), lse.zero_()
    g.replay()
    torch.cuda.synchronize()
    R.check_attention(p, out, lse, R.attention(p))
    assert (filler == 0x7f).all()
    del g
    ctx.close()


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 bytes and 2^31 elements per array; the request's pages lie at its end."""
    p = R.Problem(lens=[500], rows=[5], hq=4, hkv=2, d=128, page=64, seed=14, pool_pages=(1 << 31) // (64 * 256) + 64)
    p.table[0, :8] = p.n_pages - 1 - np.arange(8)
    check(p)


def test_lse_and_status_are_optional():
    p = R.Problem(lens=[90], rows=[4], hq=4, hkv=2, d=64, page=16, seed=15).fill().device()
    ctx, out = p.context(), torch.zeros_like(p.q)
    ctx.hvd_attn_paged(1, p.cache(), p.t_len, p.t_off, 0, p.total, None, None, p.q, out)
    R.check_attention(p, out, None, R.attention(p))
    ctx.close()


@pytest.mark.parametrize("seed", range(40))
def test_random_batches(seed):
    rng = np.random.default_rng(1000 + seed)
    B = int(rng.integers(1, 12))
    tree = bool(rng.random() < 0.4)
    hkv = int(rng.integers(1, 5))
    g = int(rng.choice([1, 2, 3, 4, 5, 8, 16]))
    most = 40 if rng.random() < 0.7 else 300
    rows = [int(x) for x in rng.integers(1, (66 if tree else most) + 1, B)]
    sel = [int(rng.integers(-1, r + 3)) for r in rows] if tree or rng.random() < 0.5 else None
    if sel is not None:
        rows = [min(r, 65) for r in rows]
    lens = [int(x) for x in np.exp(rng.uniform(0, np.log(6000), B)) - 1]
    check(R.Problem(lens=lens, rows=rows, sel=sel, hq=g * hkv, hkv=hkv, d=int(rng.choice([32, 64, 80, 128, 128])),
                    page=int(rng.choice([8, 16, 32, 56, 64, 256])), dtype=BF if rng.random() < 0.7 else HF, tree=True if tree else None,
                    bad=0.05, order=str(rng.choice(["slots", "heads"])), seed=seed))


def test_refusals():
    import paper_2606_01019_b200 as H
    p = R.Problem(lens=[20], rows=[4], hq=4, hkv=2, d=64, page=16).fill().device()
    plain = H.Context(max_batch=1, k_cap=4, max_hist_len=16, max_rows=4, max_vocab=8)
    out, lse = torch.zeros_like(p.q), torch.zeros(p.total, p.hq, device="cuda")
    args = lambda **o: [o.get("B", 1), o.get("cache") or p.cache(), p.t_len, p.t_off, 0, o.get("rows", p.total), o.get("sel"), o.get("par"),
                        o.get("q", p.q), o.get("out", out), lse, p.status]

    def refused(ctx, text, **o):
        with pytest.raises(H.HvdError, match=text):
            ctx.hvd_attn_paged(*args(**o))
    refused(plain, "hvd_set_attention first")
    plain.close()
    ctx = p.context()
    refused(ctx, "B outside", B=0)
    refused(ctx, "B outside", B=2)
    refused(ctx, "parent needs sel_len", par=torch.zeros(1, 64, dtype=torch.int32, device="cuda"))
    refused(ctx, "another array", out=p.q)
    refused(ctx, "total_rows", rows=p.total + 1, q=torch.zeros(9, 4, 64, dtype=BF, device="cuda"), out=torch.zeros(9, 4, 64, dtype=BF, device="cuda"))
    refused(ctx, "16-byte aligned", q=torch.zeros(4 * 256 + 4, dtype=BF, device="cuda")[4:].reshape(4, 4, 64))
    refused(ctx, "multiples of 8", q=torch.zeros(4, 4, 68, dtype=BF, device="cuda")[..., :64])
    refused(ctx, "another type", q=p.q.half())
    refused(ctx, "n_q_heads", q=torch.zeros(4, 8, 64, dtype=BF, device="cuda"))
    odd = torch.zeros(4, 12, 2, 64, dtype=BF, device="cuda")
    refused(ctx, "page_size", cache=H.KvCache(odd, odd.clone(), p.t_table))
    for bad in (dict(head_dim=136), dict(head_dim=60), dict(n_q_heads=5), dict(n_q_heads=0), dict(dtype=H.F32), dict(rot_dim=3),
                dict(rot_dim=66), dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")), dict(rope_base=1.0), dict(rot_layout=2),
                dict(rope_scaling=9), dict(rope_scaling=H.ROPE_LINEAR, rope_factor=0.5), dict(rope_scaling=H.ROPE_PARTS, rope_factor=2.0),
                dict(n_q_heads=258, n_kv_heads=2)):
        with pytest.raises(H.HvdError, match="hvd_set_attention"):
            p.context(**bad)
    # what was set stays usable after a refusal, and a new geometry takes the old one's place
    with pytest.raises(H.HvdError):
        ctx.hvd_set_attention(n_q_heads=4, n_kv_heads=3, head_dim=64)
    ctx.hvd_attn_paged(*args())
    R.check_attention(p, out, lse, R.attention(p))
    ctx.close()


def test_arrays_too_small_for_the_call_are_refused():
    import paper_2606_01019_b200 as H
    p = R.Problem(lens=[20, 9], rows=[4, 4], hq=4, hkv=2, d=64, page=16).fill().device()
    ctx, out = p.context(), torch.zeros_like(p.q)
    lse = torch.zeros(p.total, p.hq, device="cuda")
    short = H.KvCache(p.k, p.v, p.t_table[:1].contiguous())
    attn = lambda cache, lse: ctx.hvd_attn_paged(2, cache, p.t_len, p.t_off, 0, p.total, None, None, p.q, out, lse)
    with pytest.raises(H.HvdError, match="page table has 1"):
        attn(short, lse)
    kv = torch.zeros(p.total, 2, 64, dtype=BF, device="cuda")
    with pytest.raises(H.HvdError, match="page table has 1"):
        ctx.hvd_rope_append(2, short, p.t_len, p.t_off, 0, p.total, None, None, p.q, kv, kv, out, p.status)
    with pytest.raises(H.HvdError, match="page table has 1"):
        ctx.hvd_kv_commit(2, short, 1, 0, p.t_len, None, None, None, None, None, p.t_len, torch.empty_like(p.t_len))
    for bad in (lse[:-1], lse.half(), torch.zeros(p.total, 2 * p.hq, device="cuda")[:, ::2]):
        with pytest.raises(H.HvdError, match="lse is a contiguous"):
            attn(p.cache(), bad)
    for i in range(3):
        with pytest.raises(H.HvdError, match="CUDA tensors"):
            H.KvCache(*[t.cpu() if i == j else t for j, t in enumerate((p.k, p.v, p.t_table))])
    attn(p.cache(), lse)
    R.check_attention(p, out, lse, R.attention(p))
    ctx.close()


def _again(env, select):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    cmd = [sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu", "tests/test_gpu_attention.py", "tests/test_gpu_rope.py",
           "tests/test_gpu_kv_commit.py", "tests/test_gpu_target_forward.py", "-k", select]
    res = subprocess.run(cmd, cwd=root, env=dict(os.environ, **env), capture_output=True, text=True, timeout=900)
    assert res.returncode == 0, res.stdout[-3000:] + res.stderr[-2000:]
    assert " passed" in res.stdout


def test_again_with_plain_launches():
    """No programmatic dependent launch: results must not depend on how far consecutive kernels overlap."""
    _again({"HVD_PDL_MASK": "0"}, "(random or trees or few_requests or decoding or rows or become) and not again")


def test_again_against_the_bounds_checked_build():
    """The build with -DHVD_DEBUG_BOUNDS: every context must close with device status 0."""
    from paper_2606_01019_b200 import build
    _again({"HVD_B200_LIB": build.build_bounds_checked(), "HVD_ASSERT_DEVICE_STATUS": "1"}, "not again")
