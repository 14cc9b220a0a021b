"""The cache operators together, as examples/target_forward.py uses them: drafts, forward on the paged cache, verification and
commit in a loop, against a plain forward of the whole histories in 64 bits."""
import numpy as np
import pytest
import torch

from examples.target_forward import Decoder, TargetModel, prompts
from tests import attn_reference as R

pytestmark = pytest.mark.gpu


def plain(model, tokens):
    """(logits [n, vocab], per layer rotated k and v [n, heads, d]) of one history, in 64 bits."""
    n = len(tokens)
    x = model.embed[torch.as_tensor(tokens, device="cuda").long()].double()
    norm = lambda y: y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)
    freq = 10000.0 ** (-2.0 * torch.arange(model.d // 2, device="cuda", dtype=torch.float64) / model.d)
    pos, kv = torch.arange(n, device="cuda"), []
    hide = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
    for i in range(model.layers):
        qkv = (norm(x) @ model.qkv[i].double().T).view(n, -1, model.d)
        q, k, v = qkv.split([model.hq, model.hkv, model.hkv], dim=1)
        q, _ = R.turned(q, pos, freq, 1.0, model.d, False)
        k, _ = R.turned(k, pos, freq, 1.0, model.d, False)
        kv.append((k, v))
        g = model.hq // model.hkv
        s = torch.einsum("rhd,nhd->hrn", q, k.repeat_interleave(g, 1)) * model.d ** -0.5
        p = s.masked_fill(hide, -torch.inf).softmax(-1)
        x = x + torch.einsum("hrn,nhd->rhd", p, v.repeat_interleave(g, 1)).reshape(n, -1) @ model.out[i].double().T
        gate, up = (norm(x) @ model.up[i].double().T).chunk(2, -1)
        x = x + (torch.nn.functional.silu(gate) * up) @ model.down[i].double().T
    return norm(x) @ model.head.double().T, kv


@pytest.mark.parametrize("tree", [False, True])
def test_decoding_with_drafts_is_greedy_decoding(tree):
    model = TargetModel()
    start = prompts(6, model.vocab, seed=3)
    dec = Decoder(model, start, new_tokens=200, tree=tree)
    best, steps = 0, 30
    for _ in range(steps):
        dec.step()
        best = max(best, int(dec.batch.accepted.max()))
        assert (dec.batch.status.cpu().numpy() == 0).all() and (dec.cache.status.cpu().numpy() == 0).all()
    assert dec.ctx.hvd_device_status() == 0
    hist = dec.histories()
    made = sum(len(h) - len(p) for h, p in zip(hist, start))
    assert best >= 2 and made > steps * 6                     # drafts were accepted, in trees off the first path
    assert (dec.cache.length.cpu().numpy() == [len(h) - 1 for h in hist]).all()
    off = 0.0
    for b, (h, p) in enumerate(zip(hist, start)):
        logits, kv = plain(model, h)
        # bfloat16 through two layers: every sum of products is rounded to 2^-8 of itself, some ten times in a row, so a logit is
        # off by a few per cent of the row's spread
        rows = logits[len(p) - 1:len(h) - 1]
        took = torch.as_tensor(h[len(p):], device="cuda").long()
        short = rows.max(-1).values - rows.gather(1, took[:, None])[:, 0]
        assert bool((short <= 0.1 * rows.std(-1)).all()), float((short / rows.std(-1)).max())
        off = max(off, float((short > 0).float().mean()))
        # what the cache holds is what a forward of the final history makes, whatever drafts passed through it
        n = len(h) - 1
        t = np.arange(n)
        pages = dec.cache.table[b, torch.as_tensor(t // 16, device="cuda")].long()
        slot = torch.as_tensor(t % 16, device="cuda")
        for i, (k, v) in enumerate(kv):
            for got, want in ((dec.cache.k, k), (dec.cache.v, v)):
                e = (got[i][pages, slot].double() - want[:n]).abs()
                assert bool((e <= 0.06 * want[:n].std()).all()), (i, float(e.max() / want[:n].std()))
    assert off < 0.2
    dec.close()
