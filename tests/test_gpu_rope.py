"""hvd_rope_append against the rotation in 64 bits; what it leaves alone stays bit for bit."""
import numpy as np
import pytest
import torch

from tests import attn_reference as R

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def positions(p):
    pos, fresh = [], []
    for b in range(p.B):
        for i in range(p.rows[b]):
            new = i < p.n_new[b]
            line = None if p.parent is None or not new else R.line_of(p.parent[b], i)
            depth = i if p.parent is None else (0 if line is None else len(line) - 1)
            pos.append(p.lens[b] + depth)
            fresh.append(new)
    return torch.tensor(pos, device="cuda"), torch.tensor(fresh, device="cuda", dtype=torch.bool)


def run(p, in_place=False, fused=True, row_off=True, **cfg):
    import paper_2606_01019_b200 as H
    p.fill(chunk=False).device()
    ctx = p.context(**cfg)
    qkv = torch.randn(p.total, p.hq + 2 * p.hkv, p.d, device="cuda").to(p.dtype)
    q, k, v = qkv.split([p.hq, p.hkv, p.hkv], dim=1)
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    was = [t.clone() for t in (q, k, v, p.k, p.v)]
    q_out = q if in_place else torch.full((p.total, p.hq, p.d), 9.0, dtype=p.dtype, device="cuda")
    ctx.hvd_rope_append(p.B, p.cache(), p.t_len, p.t_off if row_off else None, p.k_uniform, p.total, p.t_sel, p.t_par, q, k, v, q_out,
                        p.status)
    torch.cuda.synchronize()
    assert ctx.hvd_device_status() == 0
    ctx.close()
    freq, mag = H.hvd_rope_frequencies(n_q_heads=p.hq, n_kv_heads=p.hkv, head_dim=p.d, **cfg)
    return was, q_out, freq, mag


def check(p, in_place=False, **kw):
    import paper_2606_01019_b200 as H
    was, q_out, freq, mag = run(p, in_place, **kw)
    q, k, v, k_pool, v_pool = was
    rot, pairs = kw.get("rot_dim", p.d), kw.get("rot_layout") == H.ROPE_PAIRS
    pos, fresh = positions(p)
    u = R.UNIT[p.dtype]
    # one rounding to the type; angle, sincos and the two products in 32 bits: together below 2^-20 of |x| + |y|
    tol = lambda y, size: u * y.abs() + 2.0 ** -20 * size + 2.0 ** -25
    wq, sq = R.turned(q, pos, freq, mag, rot, pairs)
    wk, sk = R.turned(k, pos, freq, mag, rot, pairs)
    assert bool(((q_out.double() - wq).abs() <= tol(wq, sq))[fresh].all())
    assert torch.equal(q_out[fresh][..., rot:], q[fresh][..., rot:])
    rest = q_out[~fresh]
    assert torch.equal(rest, q[~fresh]) if in_place else bool((rest == 9).all())
    got_k, got_v = p.k.clone(), p.v.clone()
    for b in range(p.B):
        m, r = p.n_new[b], int(p.off[b])
        if m:
            at = p.places(b, p.lens[b], p.lens[b] + m)
            e = (got_k[at].double() - wk[r:r + m]).abs()
            assert bool((e <= tol(wk[r:r + m], sk[r:r + m])).all()), float(e.max())
            assert torch.equal(got_k[at][..., rot:], k[r:r + m][..., rot:])
            assert torch.equal(got_v[at], v[r:r + m])
            got_k[at], got_v[at] = k_pool[at], v_pool[at]
    bits = lambda t: t.contiguous().view(torch.int16)
    assert torch.equal(bits(got_k), bits(k_pool)) and torch.equal(bits(got_v), bits(v_pool))   # nothing else was written
    assert (p.status == 0).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("pairs", [0, 1])
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 64), (64, 64), (80, 80), (96, 32), (64, 20), (128, 2), (72, 6), (64, 0), (8, 8), (120, 60)])
def test_layouts_and_partial_heads(d, rot, pairs, dtype):
    check(R.Problem(lens=[0, 17, 300], rows=[5, 1, 9], hq=6, hkv=2, d=d, page=16, dtype=dtype, seed=d + rot), rot_dim=rot, rot_layout=pairs)


@pytest.mark.parametrize("cfg", [dict(rope_scaling=1, rope_factor=4.0), dict(rope_scaling=2, rope_factor=8.0, rope_base=500000.0),
                                 dict(rope_scaling=3, rope_factor=32.0, rope_original_len=4096.0, rope_low=1.0, rope_high=32.0, rope_magnitude=1.3466),
                                 dict(rope_scaling=4, rope_factor=8.0, rope_original_len=8192.0, rope_low=1.0, rope_high=4.0),
                                 dict(rope_magnitude=0.5)])
@pytest.mark.parametrize("pairs", [0, 1])
def test_scalings(cfg, pairs):
    check(R.Problem(lens=[5000, 3], rows=[9, 40], hq=8, hkv=4, d=128, page=32, seed=pairs), rot_layout=pairs, **cfg)


def test_positions_far_out():
    """Beyond 2^24 a 32-bit float no longer holds every position."""
    p = R.Problem(lens=[(1 << 24) + 1, 1_000_003], rows=[3, 5], hq=4, hkv=1, d=64, page=65536, seed=3, table_extra=0)
    p.fill = lambda chunk=True: p
    check(p)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (32, 8), (3, 1), (128, 1), (20, 20)])
@pytest.mark.parametrize("rows", [1, 2, 33, 700])
def test_heads_and_rows(hq, hkv, rows):
    check(R.Problem(lens=[10, 0, 99], rows=[rows, 1, rows], hq=hq, hkv=hkv, d=64, page=24, order="heads", seed=hq))


@pytest.mark.parametrize("B", [1, 2, 255, 256, 257, 300, 1000])
def test_batches_of_ragged_chunks(B):
    rng = np.random.default_rng(B)
    check(R.Problem(lens=[int(x) for x in rng.integers(0, 60, B)], rows=[int(x) for x in rng.integers(0, 5, B)] if B > 1 else [3], hq=2, hkv=1, d=64,
                    page=16, seed=B))


def test_in_place_and_separate_inputs():
    kw = dict(lens=[77, 5], rows=[9, 9], sel=[4, 8], k_cap=8, hq=8, hkv=2, d=128, page=16, uniform=True)
    check(R.Problem(**kw), in_place=True)
    check(R.Problem(**kw), fused=False, row_off=False)


def test_trees_turn_by_depth():
    check(R.Problem(lens=[1000, 3, 0], rows=[33, 65, 10], sel=[32, 64, 5], hq=4, hkv=2, d=64, page=16, tree=True, bad=0.1, seed=7))


def test_unusable_requests_and_pages():
    p = R.Problem(lens=[20, 20, 30], rows=[4, 5, 6], hq=4, hkv=2, d=64, page=16, seed=6).fill(chunk=False)
    p.lens[1] = -3
    p.table[2, 2] = p.n_pages                                   # tokens 32..35 have no page
    p.device()
    ctx = p.context()
    x = torch.randn(p.total, p.hq + 2 * p.hkv, p.d, device="cuda").to(BF)
    q, k, v = x.split([4, 2, 2], dim=1)
    before, q_out = p.v.clone(), torch.full((p.total, 4, 64), 9.0, dtype=BF, device="cuda")
    ctx.hvd_rope_append(p.B, p.cache(), p.t_len, p.t_off, 0, p.total, None, None, q, k, v, q_out, p.status)
    assert p.status.tolist() == [0, 2, 3]
    assert (q_out[4:9] == 9).all() and (q_out[:4] != 9).any(1).all() and (q_out[9:] != 9).any(1).all()
    for b, lo, hi, r in ((0, 20, 24, 0), (2, 30, 32, 9)):
        at = p.places(b, lo, hi)
        assert torch.equal(p.v[at], v[r:r + hi - lo])
        before[at] = p.v[at]
    assert torch.equal(before.view(torch.int16), p.v.view(torch.int16))
    assert ctx.hvd_device_status() == 0
    ctx.close()


@pytest.mark.parametrize("off,total", [([0, 4, -7, 15, 20], 20), ([0, 100, 200, 4, 8, 12], 12), ([30, -1, 0, 5, 9], 9), ([0, 3, 3, 99, 9, 20], 20), (600, None),
                                       (2000, None)])
def test_requests_beside_bad_offsets_are_appended(off, total):
    """Offsets that run backwards or leave the rows spoil the requests that they bound and no others."""
    rng = np.random.default_rng(9)
    if total is None:
        rows = rng.integers(0, 4, off)
        off = np.concatenate([[0], np.cumsum(rows)])
        total = int(off[-1])
        off[rng.choice(len(off) - 2, 40, replace=False) + 1] = rng.choice([-5, total + 1, 1 << 40, -(1 << 40)], 40)
    off = np.asarray(off, np.int64)
    B = len(off) - 1
    p = R.Problem(lens=[int(x) for x in rng.integers(0, 40, B)], rows=[24] * B, hq=2, hkv=1, d=64, page=16, seed=B).device()
    p.k.zero_(), p.v.zero_()
    ctx = p.context()
    x = torch.rand(total, 4, 64, device="cuda").to(BF) + 1
    q, k, v = x.split([2, 1, 1], dim=1)
    q_out = torch.full((total, 2, 64), 9.0, dtype=BF, device="cuda")
    t_off = torch.as_tensor(off, device="cuda")
    ctx.hvd_rope_append(B, p.cache(), p.t_len, t_off, 0, total, None, None, q, k, v, q_out, p.status)
    good = (off[:-1] >= 0) & (off[1:] <= total) & (off[1:] >= off[:-1])
    assert p.status.tolist() == [0 if g else 2 for g in good] and 0 < good.sum() < B
    want, written = torch.zeros_like(p.v), np.zeros(total, bool)
    for b in np.nonzero(good)[0]:
        written[off[b]:off[b + 1]] = True
        at = p.places(b, p.lens[b], p.lens[b] + int(off[b + 1] - off[b]))
        want[at] = v[off[b]:off[b + 1]]
    assert torch.equal(want, p.v)
    up = torch.as_tensor(written, device="cuda")
    assert (q_out[~up] == 9).all() and (q_out[up] != 9).any(2).all()
    assert ctx.hvd_device_status() == 0
    ctx.close()


def test_offsets_beyond_32_bits():
    p = R.Problem(lens=[500], rows=[5], hq=4, hkv=2, d=128, page=64, seed=14, pool_pages=(1 << 31) // (64 * 256) + 64)
    p.table[0, :8] = p.n_pages - 1 - np.arange(8)
    check(p)


def test_refusals():
    import paper_2606_01019_b200 as H
    p = R.Problem(lens=[20], rows=[4], hq=4, hkv=2, d=64, page=16).device()
    ctx = p.context()
    k = torch.zeros(4, 2, 64, dtype=BF, device="cuda")
    call = lambda q=p.q, k=k, v=k, out=torch.zeros_like(p.q), B=1, par=None: ctx.hvd_rope_append(
        B, p.cache(), p.t_len, p.t_off, 0, p.total, None, par, q, k, v, out, p.status)
    call()
    for text, kw in (("B outside", dict(B=7)), ("parent needs sel_len", dict(par=p.t_len)), ("n_kv_heads", dict(k=p.q)),
                     ("same strides", dict(q=torch.zeros(4, 8, 64, dtype=BF, device="cuda")[:, :4], out=None)),
                     ("another type", dict(v=k.half()))):
        if kw.get("out", 0) is None:
            kw["out"] = torch.as_strided(kw["q"], (4, 4, 64), (256, 64, 1))
        with pytest.raises(H.HvdError, match=text):
            call(**kw)
    ctx.close()
