"""The cache operators of a target forward over drafted tokens, as workloads with a plain form.

Three operators, each called once per ``run``:

* ``rope``   rotary positions on the chunk's queries and keys, keys and values appended to the paged cache
  (``Context.hvd_rope_append``);
* ``attn``   attention of the chunk's rows over the paged cache (``Context.hvd_attn_paged``);
* ``commit`` the accepted path of a token tree moved behind the cached tokens, in every layer
  (``Context.hvd_kv_commit``).

A chunk is what one decoding step hands to the target model: per request the last committed token (the
root) and its draft, or a piece of a prompt.  ``own`` chooses between the library's kernels and the plain
form, elementary torch operations in 32 bits.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ---------------------------------------------------------------- cases

def listed():
    return [
        # one request, one token, an odd context: the smallest call a chat step makes, pure latency
        dict(name="attn one token", op="attn", B=1, lo=1037, hi=1037, rows=1, hq=32, hkv=8, d=128, page=16, dtype="bf16",
             tree=False, order="slots"),
        # four requests of 2 K tokens with a draft of 8: the smallest verification step of the benchmark
        dict(name="attn verify 4x2K", op="attn", B=4, lo=2048, hi=2048, rows=9, hq=32, hkv=8, d=128, page=16, dtype="bf16",
             tree=False, order="slots"),
        # plain decode of a ragged batch (requests without a draft): single-token form, bandwidth-bound
        dict(name="attn decode ragged", op="attn", B=96, lo=512, hi=32768, rows=1, hq=32, hkv=8, d=128, page=64,
             dtype="f16", tree=False, order="slots"),
        # 64 requests of 16 K tokens with a draft of 16: the benchmark's middle workload
        dict(name="attn verify 64x16K", op="attn", B=64, lo=16384, hi=16384, rows=17, hq=32, hkv=8, d=128, page=32,
             dtype="bf16", tree=False, order="heads"),
        # token trees of 32 nodes, ragged contexts, narrow heads: the model drafter's shape
        dict(name="attn tree ragged", op="attn", B=32, lo=512, hi=65536, rows=33, hq=32, hkv=4, d=64, page=16, dtype="bf16",
             tree=True, order="slots"),
        # 128 K contexts with a draft of 64 on one rank's share of the heads: 520 rows a head, matrix-bound
        dict(name="attn verify 8x128K", op="attn", B=8, lo=131072, hi=131072, rows=65, hq=16, hkv=2, d=128, page=64,
             dtype="bf16", tree=False, order="slots"),
        # a piece of a prompt behind cached tokens, odd sizes: matrix-bound
        dict(name="attn prompt piece", op="attn", B=4, lo=1500, hi=9000, rows=2047, hq=32, hkv=8, d=128, page=32,
             dtype="bf16", tree=False, order="slots"),
        # the rotary step of the smallest verification
        dict(name="rope verify 4x2K", op="rope", B=4, lo=2048, hi=2048, rows=9, hq=32, hkv=8, d=128, page=16, dtype="bf16",
             tree=False, order="slots", rot=128, pairs=False, scaling="plain"),
        # trees far into long contexts, positions stretched by parts of the spectrum
        dict(name="rope tree long", op="rope", B=16, lo=30000, hi=131072, rows=65, hq=16, hkv=2, d=128, page=64,
             dtype="bf16", tree=True, order="slots", rot=128, pairs=False, scaling="parts"),
        # a piece of a prompt, interleaved pairs, half of each head rotated
        dict(name="rope prompt piece", op="rope", B=4, lo=1500, hi=9000, rows=2047, hq=32, hkv=8, d=128, page=32,
             dtype="f16", tree=False, order="heads", rot=64, pairs=True, scaling="linear"),
        # trees of 32 nodes, one layer's call for every layer of a small model
        dict(name="commit 16 trees", op="commit", B=16, lo=700, hi=900, rows=33, hq=32, hkv=8, d=128, page=16, dtype="bf16",
             tree=True, order="slots", layers=16, k_cap=64),
        # a large ragged batch, many layers, narrow heads
        dict(name="commit 128 trees", op="commit", B=128, lo=128, hi=1024, rows=33, hq=32, hkv=4, d=64, page=32,
             dtype="bf16", tree=True, order="heads", layers=32, k_cap=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "rope", "rope", "commit"])
    g, hkv = rng.choice([1, 2, 3, 4, 5, 7, 8, 16]), rng.choice([1, 2, 4, 8])
    d = rng.choice([64, 80, 96, 128, 128])
    c = dict(op=op, hq=g * hkv, hkv=hkv, d=d, page=rng.choice([8, 16, 16, 24, 32, 48, 64, 128, 256]),
             dtype=rng.choice(["bf16", "bf16", "f16"]), tree=rng.random() < 0.3, order=rng.choice(["slots", "heads"]))
    if op == "attn":
        kind = rng.choice(["decode", "draft", "draft", "draft", "prompt"])
        if kind == "prompt":
            # the listed piece of a prompt has 2.9e9 pairs of a row and a key over its heads
            c.update(tree=False, rows=_log(rng, 100, 2048))
            c["B"] = _log(rng, 1, max(1, min(4, int(2.5e9) // (c["hq"] * c["rows"] * (c["rows"] + 64)))))
            c["hi"] = _log(rng, 16, min(9000, int(2.5e9) // (c["B"] * c["hq"] * c["rows"]) - c["rows"]))
        else:
            c.update(rows=1 if kind == "decode" else rng.randint(2, 65), B=_log(rng, 1, 128))
            # contexts as long as the largest listed case's work allows
            most = min(131072, int(1 << 20) * 8 * 128 // (c["B"] * hkv * d), int(5e11) // (c["B"] * c["rows"] * 4 * c["hq"] * d))
            c["hi"] = _log(rng, 256, max(257, most))
        c["lo"] = max(1, int(c["hi"] / rng.choice([1, 1, 4, 32])))
    elif op == "rope":
        c.update(rot=rng.choice([d, d, d // 2]), pairs=rng.random() < 0.5,
                 scaling=rng.choice(["plain", "linear", "base", "parts", "bands"]))
        if rng.random() < 0.4:
            c.update(tree=False, rows=_log(rng, 100, 2048), B=_log(rng, 1, 4), hi=_log(rng, 16, 9000))
        else:
            c.update(rows=rng.randint(1, 65), B=_log(rng, 1, 128))
            c["hi"] = _log(rng, 64, max(65, min(131072, int(1 << 19) * 8 * 128 // (c["B"] * hkv * d))))
        c["lo"] = max(1, c["hi"] // rng.choice([1, 4]))
    else:
        c.update(tree=True, rows=rng.randint(2, 65), B=_log(rng, 4, 160), layers=_log(rng, 4, 40), k_cap=64)
        c["hi"] = _log(rng, 100, max(101, min(1024, int(1 << 19) * 8 * 128 // (c["B"] * hkv * d * c["layers"]))))
        c["lo"] = max(1, c["hi"] // rng.choice([1, 4]))
    return c


# ---------------------------------------------------------------- what follows from a case alone

def _lens(c):
    """Tokens cached before the chunk, per request: log-uniform between lo and hi, in no order."""
    r = random.Random("%s %s %s" % (c["B"], c["lo"], c["hi"]))
    n = [int(round(c["lo"] * (c["hi"] / c["lo"]) ** ((i + 0.5) / c["B"]))) for i in range(c["B"])]
    r.shuffle(n)
    return n


def _trees(c, most_depth=8, most_children=4):
    """Parents of every request's nodes: -1 (under the root) or an earlier node."""
    r = random.Random("tree %s %s" % (c["B"], c["rows"]))
    par = []
    for _ in range(c["B"]):
        p, depth, kids = [], [], {}
        for i in range(c["rows"] - 1):
            while True:
                j = r.randint(-1, i - 1)
                if kids.get(j, 0) < most_children * (2 if j < 0 else 1) and (j < 0 or depth[j] < most_depth):
                    break
                if all(kids.get(j, 0) >= most_children * (2 if j < 0 else 1) or (j >= 0 and depth[j] >= most_depth)
                       for j in range(-1, i)):
                    j = -1
                    break
            kids[j] = kids.get(j, 0) + 1
            p.append(j)
            depth.append(1 if j < 0 else depth[j] + 1)
        par.append(p)
    return par


def _path(par, r):
    """A path from the root: what verification accepts."""
    kids = [j for j, p in enumerate(par) if p < 0]
    path = []
    while kids and r.random() < 0.8:
        path.append(r.choice(kids))
        kids = [j for j, p in enumerate(par) if p == path[-1]]
    return path


def _paths(c):
    r = random.Random("path %s %s" % (c["B"], c["rows"]))
    return [_path(p, r) for p in _trees(c)]


def work(c):
    n, d, h = c["B"] * c["rows"], c["d"], 2 * c["d"]
    if c["op"] == "attn":
        keys = sum(_lens(c)) + n
        if c["tree"]:
            seen = sum(l * c["rows"] for l in _lens(c)) + 2 * n  # at least the root and itself
        else:
            seen = sum(l * c["rows"] for l in _lens(c)) + c["B"] * c["rows"] * (c["rows"] + 1) // 2
        return {"bytes": 2 * keys * c["hkv"] * h + 2 * n * c["hq"] * h + 4 * n * c["hq"], "flops": 4 * seen * c["hq"] * d}
    if c["op"] == "rope":
        return {"bytes": 2 * n * (c["hq"] + 2 * c["hkv"]) * h, "flops": 3 * n * (c["hq"] + c["hkv"]) * c["rot"]}
    moved = sum(sum(node != j for j, node in enumerate(p)) for p in _paths(c))
    return {"bytes": 2 * c["layers"] * moved * 2 * c["hkv"] * h + 4 * c["B"] * (2 * c["rows"] + 4), "flops": 0}


# ---------------------------------------------------------------- inputs

class State:
    pass


def _rope_numbers(c):
    """Angular frequency per rotated pair (64 bits) and the factor on cos and sin."""
    rot, base, original = c["rot"], 10000.0, 4096.0
    i = np.arange(rot // 2, dtype=np.float64)
    w = base ** (-2.0 * i / rot)
    if c["scaling"] == "linear":
        return w / 4.0, 1.0
    if c["scaling"] == "base":
        return (base * 8.0 ** (rot / (rot - 2.0))) ** (-2.0 * i / rot), 1.0
    turns = original * w / (2.0 * math.pi)  # turns within the original context
    if c["scaling"] == "parts":  # whole turns kept, slow ones stretched 32 times, a ramp over the index between
        edge = lambda t: rot * math.log(original / (t * 2.0 * math.pi)) / (2.0 * math.log(base))
        lo, hi = max(math.floor(edge(32.0)), 0.0), min(math.ceil(edge(1.0)), rot - 1.0)
        keep = 1.0 - np.clip((i - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        return w * keep + (w / 32.0) * (1.0 - keep), 0.1 * math.log(32.0) + 1.0
    if c["scaling"] == "bands":  # the same with the ramp over the number of turns
        keep = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return w * keep + (w / 8.0) * (1.0 - keep), 1.0
    return w, 1.0


_ROPE_ARGS = {  # the same numbers as a user names them to the library
    "plain": dict(), "linear": dict(rope_factor=4.0), "base": dict(rope_factor=8.0),
    "parts": dict(rope_factor=32.0, rope_original_len=4096.0, rope_low=1.0, rope_high=32.0, rope_magnitude=0.1 * math.log(32.0) + 1.0),
    "bands": dict(rope_factor=8.0, rope_original_len=4096.0, rope_low=1.0, rope_high=4.0)}


def prepare(case, seed):
    c, s = dict(case), State()
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    B, rows, hkv, hq, d, ps = (c[k] for k in ("B", "rows", "hkv", "hq", "d", "page"))
    t = DTYPES[c["dtype"]]
    randn = lambda *sh: torch.randn(*sh, generator=g, device=DEV, dtype=torch.float32 if math.prod(sh) < 1 << 24 else t).to(t)
    lens = _lens(c)
    need = [-(-(n + rows) // ps) for n in lens]
    s.c, s.pages = c, sum(need) + 3
    width = max(need)
    # the pool's pages belong to the requests in no order
    perm = torch.randperm(s.pages, generator=g, device=DEV).to(torch.int32)
    off = torch.tensor(np.concatenate([[0], np.cumsum(need)[:-1]]), device=DEV)
    col = torch.arange(width, device=DEV)
    held = col[None, :] < torch.tensor(need, device=DEV)[:, None]
    s.table = torch.where(held, perm[(off[:, None] + col).clamp(max=s.pages - 1)], -1).to(torch.int32)
    s.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s.longest = max(lens) + rows
    s.total = B * rows
    s.row_off = torch.arange(B + 1, dtype=torch.int64, device=DEV) * rows
    layers = c.get("layers", 1)
    shape = (layers, s.pages, ps, hkv, d) if c["order"] == "slots" else (layers, s.pages, hkv, ps, d)
    s.k, s.v = randn(*shape), randn(*shape)
    if c["order"] == "heads":  # seen as [layer, page, slot, head, d] whatever the order in memory
        s.k, s.v = s.k.transpose(2, 3), s.v.transpose(2, 3)
    k_cap = c.get("k_cap", max(1, rows - 1) if c["tree"] else 1)
    s.k_cap = k_cap
    if c["tree"]:
        par = np.full((B, k_cap), -1, np.int32)
        par[:, :rows - 1] = _trees(c)
        s.parent = torch.tensor(par, device=DEV)
        s.n_draft = torch.full((B,), rows - 1, dtype=torch.int32, device=DEV)
    else:
        s.parent = s.n_draft = None
    if c["op"] == "attn":
        s.q = randn(s.total, hq, d) * 2  # some rows look at few keys, some at many
    elif c["op"] == "rope":
        s.qkv = randn(s.total, hq + 2 * hkv, d)  # the fused projection's output
        s.q_out = torch.empty(s.total, hq, d, dtype=t, device=DEV)
    else:
        tok = torch.randint(0, 1 << 30, (B, k_cap), generator=g, device=DEV, dtype=torch.int32)
        s.sel_draft = tok
        paths = _paths(c)
        com = torch.full((B, k_cap + 1), -1, dtype=torch.int32, device=DEV)
        flat = torch.tensor([(b, j, p) for b, path in enumerate(paths) for j, p in enumerate(path)], device=DEV).reshape(-1, 3)
        com[flat[:, 0], flat[:, 1]] = tok[flat[:, 0], flat[:, 2]]
        s.accepted = torch.tensor([len(p) for p in paths], dtype=torch.int32, device=DEV)
        com[torch.arange(B, device=DEV), s.accepted.long()] = torch.randint(0, 1 << 30, (B,), generator=g, device=DEV, dtype=torch.int32)
        s.committed, s.n_commit = com, s.accepted + 1
        s.new_len = torch.empty(B, dtype=torch.int32, device=DEV)
        s.deepest = max(len(p) for p in paths)
    if c["op"] == "rope":
        s.freq, s.mag = _rope_numbers(c)
        s.freq32 = torch.tensor(s.freq, dtype=torch.float32, device=DEV)
    if own:
        _handle(s)
    return s


def _handle(s):
    """What a serving program holds for its whole life: the context, its attention set-up, the output arrays."""
    import paper_2606_01019_b200 as H
    c = s.c
    s.H = H
    s.ctx = H.Context(max_batch=c["B"], k_cap=s.k_cap, max_hist_len=s.longest, max_rows=s.total, max_vocab=32)
    kw = dict(rot_dim=c["rot"], rot_layout=H.ROPE_PAIRS if c["pairs"] else H.ROPE_HALVES, rope_base=10000.0,
              rope_scaling={"plain": H.ROPE_PLAIN, "linear": H.ROPE_LINEAR, "base": H.ROPE_BASE, "parts": H.ROPE_PARTS,
                            "bands": H.ROPE_BANDS}[c["scaling"]], **_ROPE_ARGS[c["scaling"]]) if c["op"] == "rope" else {}
    s.ctx.hvd_set_attention(n_q_heads=c["hq"], n_kv_heads=c["hkv"], head_dim=c["d"],
                            dtype=H.BF16 if c["dtype"] == "bf16" else H.F16, **kw)
    s.cache = H.KvCache(s.k[0], s.v[0], s.table)
    s.status = torch.empty(c["B"], dtype=torch.int32, device=DEV)
    if c["op"] == "attn":
        s.out, s.lse = torch.empty_like(s.q), torch.empty(s.total, c["hq"], device=DEV)


# ---------------------------------------------------------------- one pass

def run(s):
    return (_OWN if own else _PLAIN)[s.c["op"]](s)


def _own_attn(s):
    s.ctx.hvd_attn_paged(s.c["B"], s.cache, s.lens, s.row_off, 0, s.total, s.n_draft, s.parent, s.q, s.out, s.lse, s.status)
    return {"out": s.out, "lse": s.lse}


def _own_rope(s):
    c = s.c
    q, k, v = s.qkv.split([c["hq"], c["hkv"], c["hkv"]], dim=1)
    s.ctx.hvd_rope_append(c["B"], s.cache, s.lens, s.row_off, 0, s.total, s.n_draft, s.parent, q, k, v, s.q_out, s.status)
    return {"q": s.q_out, "k": s.k[0], "v": s.v[0]}


def _own_commit(s):
    c = s.c
    s.ctx.hvd_kv_commit(c["B"], s.cache, c["layers"], s.k.stride(0), s.lens, s.parent, s.sel_draft, s.n_draft, s.accepted,
                        s.committed, s.n_commit, s.new_len)
    return {"k": s.k, "v": s.v, "len": s.new_len}


def _ancestors(parent, n):
    """seen[b, i, j]: row j of the chunk (0 the root, j the node j - 1) is row i itself or above it."""
    B = parent.shape[0]
    eye = torch.eye(n, device=DEV)
    step = eye.expand(B, n, n).clone()
    step[:, 0, 0] = 1
    up = torch.zeros(B, n, n, device=DEV).scatter_(2, torch.cat([torch.zeros(B, 1, 1, device=DEV), parent[:, :n - 1, None] + 1], 1).long(), 1.0)
    reach = torch.maximum(step, up)
    for _ in range(max(1, (n - 1).bit_length())):  # paths of 1, 2, 4, ... steps
        reach = torch.matmul(reach, reach).clamp(max=1.0)
    return reach > 0


def _plain_attn(s):
    c = s.c
    B, R, hkv, d = c["B"], c["rows"], c["hkv"], c["d"]
    pos = torch.arange(s.longest, device=DEV)
    page = s.table[:, pos // c["page"]].long().clamp(min=0)
    k = s.k[0][page, pos % c["page"]].float().permute(0, 2, 1, 3)  # [B, hkv, L, d]
    v = s.v[0][page, pos % c["page"]].float().permute(0, 2, 1, 3)
    q = s.q.float().reshape(B, R, hkv, -1, d).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, d)
    x = torch.matmul(q, k.transpose(2, 3)).reshape(B, hkv, -1, R, s.longest)
    row = pos - s.lens[:, None]  # which row of the chunk a key is: below 0 before it
    seen = row[:, None, :] <= torch.arange(R, device=DEV)[:, None]
    if s.parent is not None:
        above = _ancestors(s.parent, R).gather(2, row.clamp(0, R - 1)[:, None, :].expand(B, R, s.longest))
        seen = (row < 0)[:, None, :] | (above & (row < R)[:, None, :])
    x = x.mul_(1.0 / math.sqrt(d)).masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(top).exp_()
    z = x.sum(-1, keepdim=True)
    o = torch.matmul(x.reshape(B, hkv, -1, s.longest), v).reshape(B, hkv, -1, R, d) / z
    back = lambda y: y.permute(0, 3, 1, 2, 4).reshape(s.total, c["hq"], -1)
    return {"out": back(o).to(s.q.dtype), "lse": back(top + torch.log(z))[..., 0].contiguous()}


def _chunk_places(s):
    """Per row of the batch: its request, its index in the chunk, its page and slot."""
    c = s.c
    at = torch.arange(s.total, device=DEV)
    b, i = at // c["rows"], at % c["rows"]
    p = s.lens[b].long() + i
    return b, i, s.table[b, p // c["page"]].long(), p % c["page"]


def _plain_rope(s):
    c = s.c
    b, i, page, slot = _chunk_places(s)
    depth = i if s.parent is None else (_ancestors(s.parent, c["rows"]).sum(2) - 1)[b, i]
    a = (s.lens[b] + depth).float()[:, None] * s.freq32
    cos, sin = torch.cos(a)[:, None] * s.mag, torch.sin(a)[:, None] * s.mag
    q, k, v = s.qkv.split([c["hq"], c["hkv"], c["hkv"]], dim=1)

    def turned(x):
        x = x.float()
        r, rest = x[..., :c["rot"]], x[..., c["rot"]:]
        if c["pairs"]:
            e, o = r[..., 0::2], r[..., 1::2]
            r = torch.stack([e * cos - o * sin, e * sin + o * cos], -1).flatten(-2)
        else:
            e, o = r.chunk(2, -1)
            r = torch.cat([e * cos - o * sin, e * sin + o * cos], -1)
        return torch.cat([r, rest], -1).to(s.qkv.dtype)

    s.k[0][page, slot] = turned(k)
    s.v[0][page, slot] = v
    return {"q": turned(q), "k": s.k[0], "v": s.v[0]}


def _plain_commit(s):
    c = s.c
    B, n = c["B"], c["rows"] - 1
    rows, nodes = torch.arange(B, device=DEV), torch.arange(n, device=DEV)
    cur = torch.full((B,), -1, dtype=torch.int32, device=DEV)
    path = []
    for j in range(s.deepest):  # the walk that verification took: the first child that carries the committed token
        on = j < s.accepted
        child = (s.parent[:, :n] == cur[:, None]) & (s.sel_draft[:, :n] == s.committed[:, j, None])
        first = torch.where(child, nodes, n).amin(1).to(torch.int32)
        cur = torch.where(on, first, cur)
        path.append(torch.where(on, first, torch.full_like(first, j)))
    node = torch.stack(path, 1).long()  # rows that do not move stay where they are
    to = s.lens[:, None].long() + 1 + torch.arange(s.deepest, device=DEV)
    fro = s.lens[:, None].long() + 1 + node
    place = lambda p: (s.table[rows[:, None], p // c["page"]].long(), p % c["page"])
    (pf, sf), (pt, st) = place(fro), place(to)
    for x in (s.k, s.v):
        x[:, pt, st] = x[:, pf, sf]
    return {"k": s.k, "v": s.v, "len": s.lens + s.n_commit}


_OWN = {"attn": _own_attn, "rope": _own_rope, "commit": _own_commit}
_PLAIN = {"attn": _plain_attn, "rope": _plain_rope, "commit": _plain_commit}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    c = s.c
    lens, table, R, ps = s.lens.tolist(), s.table.cpu().numpy(), c["rows"], c["page"]
    par = None if s.parent is None else s.parent.cpu().numpy()

    def lineage(b, i):  # the chunk rows that row i descends from, itself first
        line = [i]
        while line[-1] > 0:
            line.append(line[-1] - 1 if par is None else int(par[b, line[-1] - 1]) + 1)
        return line

    if c["op"] == "attn":
        out = torch.empty(s.total, c["hq"], c["d"], dtype=torch.float64, device=DEV)
        lse = torch.empty(s.total, c["hq"], dtype=torch.float64, device=DEV)
        group = c["hq"] // c["hkv"]
        for b in range(c["B"]):
            n = lens[b] + R
            at = torch.tensor(table[b, :-(-n // ps)], device=DEV).long()
            hide = torch.ones(R, n, dtype=torch.bool, device=DEV)
            hide[:, :lens[b]] = False
            if par is None:
                hide[:, lens[b]:] = torch.ones(R, R, dtype=torch.bool, device=DEV).triu(1)
            else:
                for i in range(R):
                    hide[i, torch.tensor(lineage(b, i), device=DEV) + lens[b]] = False
            for h in range(c["hkv"]):
                k = s.k[0][at, :, h].reshape(-1, c["d"])[:n].double()
                v = s.v[0][at, :, h].reshape(-1, c["d"])[:n].double()
                for h2 in range(h * group, (h + 1) * group):
                    x = (s.q[b * R:(b + 1) * R, h2].double() @ k.T) * c["d"] ** -0.5
                    x[hide] = -math.inf
                    y = torch.logsumexp(x, 1)
                    lse[b * R:(b + 1) * R, h2] = y
                    out[b * R:(b + 1) * R, h2] = torch.exp(x - y[:, None]) @ v
        return {"out": out, "lse": lse}
    if c["op"] == "rope":
        x = s.qkv.double()
        pos = torch.tensor([lens[b] + (i if par is None else len(lineage(b, i)) - 1) for b in range(c["B"]) for i in range(R)],
                           dtype=torch.float64, device=DEV)
        angle = pos[:, None, None] * torch.tensor(s.freq, device=DEV)
        turn = torch.polar(torch.full_like(angle, s.mag), angle)
        half = c["rot"] // 2
        first = slice(0, c["rot"], 2) if c["pairs"] else slice(0, half)
        second = slice(1, c["rot"], 2) if c["pairs"] else slice(half, c["rot"])
        heads = c["hq"] + c["hkv"]
        y = torch.complex(x[:, :heads, first], x[:, :heads, second]) * turn
        x[:, :heads, first], x[:, :heads, second] = y.real, y.imag
        k, v = s.k[0].double(), s.v[0].double()
        for b in range(c["B"]):
            p = np.arange(lens[b], lens[b] + R)
            at, slot = torch.tensor(table[b, p // ps], device=DEV).long(), torch.tensor(p % ps, device=DEV)
            k[at, slot] = x[b * R:(b + 1) * R, c["hq"]:heads]
            v[at, slot] = x[b * R:(b + 1) * R, heads:]
        return {"q": x[:, :c["hq"]].contiguous(), "k": k, "v": v}
    # the moved rows are copies: their values have no rounding of their own
    k, v = s.k.clone(), s.v.clone()
    for b, path in enumerate(_paths(c)):
        for j, node in enumerate(path):
            to, fro = lens[b] + 1 + j, lens[b] + 1 + node
            for x in (k, v):
                x[:, int(table[b, to // ps]), to % ps] = x[:, int(table[b, fro // ps]), fro % ps]
    return {"k": k.double(), "v": v.double(), "len": s.lens + s.n_commit}
