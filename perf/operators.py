"""Operators of decoding with a long or bounded key-value cache, as measured workloads.

A case is one call of an operator through the public entry points of
`paper_2512_21857_amd.runtime` (`own` true), or the same operator in elementary torch
operations (`own` false).  The operators belong together: rows are rotated and appended to a
cache, attention reads all of it or the blocks that a score selects, the attention weights
that every cached slot received are accumulated, and slots of little weight are evicted.

Kinds
  rope     rotary positions of a batch of rows (queries and keys), keys and values appended
  keys     the mean key of each block of cache slots, all blocks or those that rows were added to
  sparse   tree attention over the blocks of the prefix that score best for each query row
  weights  tree attention that also adds up the weight each cache slot received
  evict    the slots of a cache that are kept under a budget, moved together in order

Shapes are those of this repository's configurations (20 heads of 64; 32 heads of 128; the
tiny fp32 model's 4 heads of 64; trees of up to 61 and 128 rows, 2352-token images) and
generic long-context ones with grouped heads (32 query heads over 8 key-value heads, 32768 and
65536 slots).
"""
import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

HALF, INTERLEAVED = "half", "interleaved"


def listed():
    return [
        # one new token of one sequence: launch latency is all there is
        dict(name="rope_decode_1", kind="rope", B=1, n=1, H=32, Hkv=32, Dh=128, rot=128, layout=HALF, scaling="plain",
             factor=1.0, orig=2416, first=2340, lo=2340, hi=2340, cap=2560, dtype="bf16", ragged=False),
        # a long prompt of a grouped-head model whose context was extended, half of each head rotated
        dict(name="rope_prompt_4096", kind="rope", B=1, n=4096, H=32, Hkv=8, Dh=128, rot=64, layout=INTERLEAVED,
             scaling="ramp", factor=16.0, orig=4096, first=61003, lo=17, hi=17, cap=4224, dtype="bf16", ragged=False),
        # the blocks that a 61-row tree was just appended to, 32 heads
        dict(name="keys_append_61", kind="keys", B=1, Hkv=32, Dh=128, block=32, lo=2401, hi=2401, cap=2560, last=61,
             dtype="bf16"),
        # every block of sixteen long caches, as after a prompt or an eviction
        dict(name="keys_rebuild_16x32k", kind="keys", B=16, Hkv=8, Dh=128, block=64, lo=20011, hi=32768, cap=32768,
             last=0, dtype="bf16"),
        # one token of one long sequence, 32 of 511 blocks: latency of a short chain of launches
        dict(name="sparse_decode_32k", kind="sparse", B=1, n=1, H=32, Hkv=8, Dh=128, block=64, sel=32, lo=32677,
             hi=32677, cap=32768, dtype="bf16", ragged=False),
        # one image's 61-row tree near its end, a third of the blocks
        dict(name="sparse_tree_61", kind="sparse", B=1, n=61, H=32, Hkv=32, Dh=128, block=32, sel=24, lo=2340, hi=2340,
             cap=2560, dtype="bf16", ragged=False),
        # sixteen long sequences with small trees, grouped heads
        dict(name="sparse_16x16_32k", kind="sparse", B=16, n=16, H=32, Hkv=8, Dh=128, block=64, sel=48, lo=8192,
             hi=32700, cap=32768, dtype="bf16", ragged=True),
        # the fp32 model's 17-row tree
        dict(name="weights_tiny_17", kind="weights", B=1, n=17, H=4, Hkv=4, Dh=64, lo=300, hi=300, cap=448, dtype="f32",
             ragged=False, decay=1.0, rated=False),
        # one token of one long sequence, grouped heads, old weight fading
        dict(name="weights_decode_64k", kind="weights", B=1, n=1, H=32, Hkv=8, Dh=128, lo=65333, hi=65333, cap=65536,
             dtype="bf16", ragged=False, decay=0.98, rated=False),
        # the ragged trees of sixteen images somewhere in theirs, rows weighted by path confidence
        dict(name="weights_16x61", kind="weights", B=16, n=61, H=32, Hkv=32, Dh=128, lo=512, hi=2400, cap=2560,
             dtype="bf16", ragged=True, decay=1.0, rated=True),
        # one layer of a long grouped-head cache to an eighth of its slots: the selection counts
        dict(name="evict_layer_64k", kind="evict", B=1, slices=8, Dh=128, lo=65321, hi=65321, cap=65536, budget=8192,
             first=4, last=256, dtype="bf16"),
        # all 32 x 32 slices of one image's cache to 1024 slots: the moving counts
        dict(name="evict_model_2400", kind="evict", B=1, slices=1024, Dh=128, lo=2400, hi=2400, cap=2560, budget=1024,
             first=4, last=128, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(32, 32, 128), (20, 20, 64), (4, 4, 64), (32, 8, 128), (16, 2, 128), (24, 8, 64), (8, 1, 64)]


def _draw(rng):
    kind = rng.choice(["rope", "keys", "sparse", "sparse", "weights", "weights", "evict"])
    H, Hkv, Dh = rng.choice(HEADS)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    B = rng.choice([1, 1, 1, 2, 3, 7, 16])
    if kind == "rope":
        Dh = rng.choice([Dh, Dh, 96])
        n, lo = _log_int(rng, 1, 4096), _log_int(rng, 1, 4096)
        return dict(kind=kind, B=B, n=n, H=H, Hkv=Hkv, Dh=Dh, rot=rng.choice([Dh, Dh, Dh // 2, 2 * rng.randint(1, Dh // 2)]),
                    layout=rng.choice([HALF, INTERLEAVED]), scaling=rng.choice(["plain", "linear", "base", "ramp"]),
                    factor=rng.choice([2.0, 8.0, 40.0]), orig=rng.choice([2048, 4096, 8192]),
                    first=_log_int(rng, 1, 1000000), lo=lo, hi=lo + rng.randint(0, 600), cap=lo + n + 600, dtype=dtype,
                    ragged=rng.random() < 0.5)
    lo = _log_int(rng, 40, 32000)
    hi = lo if B == 1 else rng.randint(lo, 32000)
    if kind == "keys":
        return dict(kind=kind, B=B, Hkv=Hkv, Dh=Dh, block=rng.choice([32, 64, 128]), lo=lo, hi=hi,
                    cap=hi + rng.randint(0, 300), last=rng.choice([0, 0, rng.randint(1, min(lo, 128))]), dtype=dtype)
    n = _log_int(rng, 1, 128)
    if kind == "sparse":
        return dict(kind=kind, B=B, n=n, H=H, Hkv=Hkv, Dh=Dh, block=rng.choice([32, 64, 128]), sel=_log_int(rng, 3, 64),
                    lo=lo, hi=hi, cap=hi + n + rng.randint(0, 300), dtype=dtype, ragged=rng.random() < 0.5)
    if kind == "weights":
        return dict(kind=kind, B=B, n=n, H=H, Hkv=Hkv, Dh=Dh, lo=lo, hi=hi, cap=hi + n + rng.randint(0, 300),
                    dtype=dtype, ragged=rng.random() < 0.5, decay=rng.choice([1.0, 0.9]), rated=rng.random() < 0.5)
    budget = _log_int(rng, 32, hi + hi // 4)
    return dict(kind=kind, B=B, slices=rng.choice([1, Hkv, 8 * Hkv, 32 * Hkv]), Dh=Dh, lo=lo, hi=hi,
                cap=hi + rng.randint(0, 300), budget=budget, first=rng.randint(0, 8), last=rng.randint(0, budget - 8),
                dtype=dtype)


def draw(rng):
    """A case of the listed ones' ranges that costs no more than the largest listed one of its kind."""
    most = {}
    for c in listed():
        w = work(c)
        most[c["kind"]] = [max(a, w[k]) for a, k in zip(most.get(c["kind"], [0, 0]), ("bytes", "flops"))]
    while True:
        c = _draw(rng)
        w = work(c)
        size = c["B"] * c.get("Hkv", c.get("slices", 1)) * c["cap"] * c["Dh"] * _esize(c)
        if w["bytes"] <= most[c["kind"]][0] and w["flops"] <= most[c["kind"]][1] and size <= 1.2e9:
            return c


def _esize(c):
    return 4 if c["dtype"] == "f32" else 2


# ------------------------------------------------------------------------------ inputs
def _gen(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000 + tag)
    return g


def _dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _normal(g, dt, *shape):
    return torch.empty(*shape, dtype=dt, device="cuda").normal_(generator=g)


def _trees(case, rng):
    """Row counts and parents of a batch's trees (rows that a draft head grew, breadth first)."""
    B, n = case["B"], case["n"]
    rows = np.full(B, n)
    if case["ragged"] and B > 1:
        rows = rng.integers(max(1, n // 4), n + 1, size=B)
        rows[0] = n
    parent = np.full((B, n), -1, dtype=np.int32)
    for b in range(B):
        for i in range(1, rows[b]):
            parent[b, i] = max(parent[b, i - 1], int(rng.integers(max(0, (i - 10) // 3), max(1, i // 2 + 1))))
            parent[b, i] = min(parent[b, i], i - 1)
    return rows.astype(np.int32), parent


def _path(parent, rows, n):
    """[n][n]: whether node j lies on the path from the root to node i; no row past `rows` sees any."""
    m = np.zeros((n, n), dtype=bool)
    for i in range(rows):
        if parent[i] >= 0:
            m[i] = m[parent[i]]
        m[i, i] = True
    return m


def _words(path):
    """[n][n] truth values -> [n][2] packed 64-bit words (bit j of row i: node j)."""
    w = np.zeros((path.shape[0], 2), dtype=np.uint64)
    for i, j in zip(*np.nonzero(path)):
        w[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return w.view(np.int64)


def _lengths(case, rng):
    L = rng.integers(case["lo"], case["hi"] + 1, size=case["B"])
    L[0] = case["hi"]
    return L.astype(np.int32)


def _inputs(case, seed):
    """What a user's program has in hand, apart from plans and workspaces."""
    kind, dt, B = case["kind"], _dtype(case), case["B"]
    rng, g = np.random.default_rng([int(seed), 7]), _gen(seed, 8)
    s = SimpleNamespace(case=case, L=_lengths(case, rng))
    s.kv_len = _dev(s.L)
    if kind == "rope":
        n, H, Hkv, Dh = (case[k] for k in ("n", "H", "Hkv", "Dh"))
        s.rows, parent = _trees(dict(case, n=min(n, 128)), rng)
        s.rows = np.maximum(1, s.rows * n // min(n, 128)).astype(np.int32)
        s.n_rows = _dev(s.rows)
        # a tree's rows share positions by depth, a prompt's follow one another
        depth = np.tile(np.arange(n, dtype=np.int32), (B, 1)) if n > 128 else np.zeros((B, n), dtype=np.int32)
        if n <= 128:
            for b in range(B):
                for i in range(1, n):
                    depth[b, i] = depth[b, parent[b, i]] + 1 if parent[b, i] >= 0 else 0
        s.pos = _dev(case["first"] + s.L[:, None] - case["lo"] + depth)
        # the three parts of one projection's output rows
        qkv = _normal(g, dt, B, n, (H + 2 * Hkv) * Dh)
        s.q = qkv[..., : H * Dh].unflatten(-1, (H, Dh))
        s.k = qkv[..., H * Dh: (H + Hkv) * Dh].unflatten(-1, (Hkv, Dh))
        s.v = qkv[..., (H + Hkv) * Dh:].unflatten(-1, (Hkv, Dh))
        s.kc = _normal(g, dt, B, Hkv, case["cap"], Dh)
        s.vc = _normal(g, dt, B, Hkv, case["cap"], Dh)
        s.out = torch.zeros(B, n, H, Dh, dtype=dt, device="cuda")
        return s
    if kind == "evict":
        S, Dh, cap = case["slices"], case["Dh"], case["cap"]
        s.kc, s.vc = _normal(g, dt, B, S, cap, Dh), _normal(g, dt, B, S, cap, Dh)
        # accumulated weight has a heavy tail, and slots that nothing attended to hold an exact zero
        w = torch.exp(2.0 * _normal(g, torch.float32, B, S, cap))
        s.w = torch.where(torch.rand(B, S, cap, generator=g, device="cuda") < 0.05, torch.zeros_like(w), w)
        keep = case["budget"]
        s.ko, s.vo = (torch.zeros(B, S, keep, Dh, dtype=dt, device="cuda") for _ in range(2))
        s.wo = torch.zeros(B, S, keep, dtype=torch.float32, device="cuda")
        s.kept = torch.full((B, S, keep), -1, dtype=torch.int32, device="cuda")
        s.new_len = torch.zeros(B, dtype=torch.int32, device="cuda")
        return s
    Hkv, Dh, cap = case["Hkv"], case["Dh"], case["cap"]
    # neighbouring keys have much in common: a direction per run of 32 slots, and noise
    s.kc = _normal(g, dt, B, Hkv, cap, Dh)
    topic = 0.7 * _normal(g, dt, B, Hkv, (cap + 31) // 32, Dh)
    whole = cap // 32 * 32
    s.kc[:, :, :whole].view(B, Hkv, whole // 32, 32, Dh).add_(topic[:, :, : whole // 32, None])
    if kind == "keys":
        n_blk = -(-cap // case["block"])
        s.start = _dev(s.L - case["last"]) if case["last"] else None
        s.out = _normal(g, torch.float32, B, Hkv, n_blk, Dh)      # means of earlier keys
        return s
    n, H = case["n"], case["H"]
    s.vc = _normal(g, dt, B, Hkv, cap, Dh)
    # the rows of one tree ask for much the same
    s.q = (_normal(g, torch.float32, B, 1, H, Dh) + 0.5 * _normal(g, torch.float32, B, n, H, Dh)).to(dt)
    s.rows, parent = _trees(case, rng)
    s.path = np.stack([_path(parent[b], s.rows[b], n) for b in range(B)])
    s.mask = _dev(np.stack([_words(p) for p in s.path]), np.int64)
    s.n_rows = _dev(s.rows)
    s.out = torch.zeros(B, n, H, Dh, dtype=dt, device="cuda")
    if kind == "sparse":
        block, n_blk = case["block"], -(-cap // case["block"])
        s.means = torch.zeros(B, Hkv, n_blk, Dh, dtype=torch.float32, device="cuda")
        for b in range(B):
            L = int(s.L[b])
            full = L // block
            s.means[b, :, :full] = s.kc[b, :, : full * block].float().view(Hkv, full, block, Dh).mean(2)
            if L % block:
                s.means[b, :, full] = s.kc[b, :, full * block: L].float().mean(1)
        s.sel = torch.full((B, n, Hkv, case["sel"]), -1, dtype=torch.int32, device="cuda")
        return s
    s.w = torch.exp(_normal(g, torch.float32, B, Hkv, cap))
    s.rating = torch.rand(B, n, generator=g, device="cuda") if case["rated"] else None
    s.wo = torch.zeros(B, Hkv, cap, dtype=torch.float32, device="cuda")
    return s


FIRST, LAST = 1, 2      # blocks at either end of the prefix that every query takes
THETA = 10000.0
FAST, SLOW = 32.0, 1.0  # turns within the original context above which a frequency stays, below which it is stretched


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        if case["kind"] == "rope":
            s.freq, s.gain = _freqs(case)
        s.paths = [_dev(p, bool) for p in s.path] if hasattr(s, "path") else None
        return s
    from paper_2512_21857_amd import runtime as rt
    kind = case["kind"]
    if kind == "rope":
        s.freq, s.gain = rt.rope_freqs(case["rot"], THETA, case["scaling"], case["factor"], case["orig"], FAST, SLOW)
    elif kind == "sparse":
        s.ws = rt.sparse_tree_attn_workspace(case["B"], case["H"], case["Hkv"], case["Dh"], case["n"], case["cap"],
                                             case["block"], case["sel"], s.q.dtype)
    elif kind == "weights":
        s.ws = rt.tree_attn_weights_workspace(case["B"], case["H"], case["Hkv"], case["Dh"], case["n"], case["cap"],
                                              s.q.dtype)
    return s


# ------------------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else PLAIN[s.case["kind"]](s)


def _run_own(s):
    from paper_2512_21857_amd import runtime as rt
    c = s.case
    kind = c["kind"]
    if kind == "rope":
        rt.rope_append(s.q, s.k, s.v, s.pos, s.kv_len, s.n_rows, s.freq, s.kc, s.vc, layout=c["layout"], gain=s.gain,
                       out=s.out)
        return {"q": s.out, "k_cache": s.kc, "v_cache": s.vc}
    if kind == "keys":
        return rt.block_keys(s.kc, s.kv_len, c["block"], start=s.start, out=s.out)
    if kind == "sparse":
        rt.sparse_tree_attn(s.q, s.kc, s.vc, s.means, s.kv_len, s.n_rows, s.n_rows, s.mask, c["cap"], c["block"],
                            c["sel"], n_first=FIRST, n_last=LAST, out=s.out, sel=s.sel, workspace=s.ws)
        return {"out": s.out, "blocks": s.sel}
    if kind == "weights":
        rt.tree_attn_weights(s.q, s.kc, s.vc, s.kv_len, s.n_rows, s.n_rows, s.mask, c["cap"], weights=s.w,
                             decay=c["decay"], row_weight=s.rating, out=s.out, weights_out=s.wo, workspace=s.ws)
        return {"out": s.out, "weights": s.wo}
    rt.kv_evict(s.kc, s.vc, s.w, s.kv_len, c["budget"], c["first"], c["last"], k_out=s.ko, v_out=s.vo,
                weights_out=s.wo, kept=s.kept, new_len=s.new_len)
    return {"k": s.ko, "v": s.vo, "weights": s.wo, "kept": s.kept, "length": s.new_len}


# ------------------------------------------------------------------------------ plain forms
def _freqs(case):
    """Radians per position of each rotated pair, and the gain of a stretched context."""
    rot, factor = case["rot"], case["factor"]
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    theta = THETA
    if case["scaling"] == "base" and rot > 2:
        theta = THETA * factor ** (rot / (rot - 2))
    f = theta ** (-2.0 * i / rot)
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "ramp":
        at = lambda turns: rot * math.log(case["orig"] / (2 * math.pi * turns)) / (2 * math.log(THETA))  # noqa: E731
        lo, hi = max(math.floor(at(FAST)), 0), min(math.ceil(at(SLOW)), rot - 1)
        t = ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return f * (1.0 - t) + f / factor * t, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _plain_rope(s):
    c, rot = s.case, s.case["rot"]
    angle = s.pos.double()[..., None] * s.freq
    cos, sin = ((f(angle) * s.gain).float()[:, :, None] for f in (torch.cos, torch.sin))

    def turn(x):
        y = x.float()
        if c["layout"] == HALF:
            a, b = y[..., : rot // 2], y[..., rot // 2: rot]
            t = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        else:
            a, b = y[..., 0:rot:2], y[..., 1:rot:2]
            t = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        return torch.cat([t, y[..., rot:]], -1).to(x.dtype)

    live = torch.arange(c["n"], device="cuda")[None] < s.n_rows[:, None]
    b, i = live.nonzero(as_tuple=True)
    slot = s.kv_len.long()[b] + i
    s.out[b, i] = turn(s.q)[b, i]
    s.kc[b, :, slot] = turn(s.k)[b, i]
    s.vc[b, :, slot] = s.v[b, i]
    return {"q": s.out, "k_cache": s.kc, "v_cache": s.vc}


def _plain_keys(s):
    c, block = s.case, s.case["block"]
    for b in range(c["B"]):
        L = int(s.L[b])
        j0 = (L - c["last"]) // block if c["last"] else 0
        full = L // block
        if full > j0:
            x = s.kc[b, :, j0 * block: full * block].float()
            s.out[b, :, j0:full] = x.view(c["Hkv"], full - j0, block, c["Dh"]).sum(2) / block
        if L % block:
            s.out[b, :, full] = s.kc[b, :, full * block: L].float().sum(1) / (L % block)
    return s.out


def _softmax_parts(q, k, see, scale):
    """Softmax of q . k over the visible keys; a row that sees none has weight zero everywhere."""
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()) * scale
    x = torch.where(see, x, torch.full_like(x, -math.inf))
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    return torch.where(total > 0, e / total, torch.zeros_like(e))


def _row_heads(x, Hkv):
    """[n][H][Dh] -> [Hkv][n * group][Dh], the query heads of one key-value head next to one another."""
    n, H, Dh = x.shape
    return x.reshape(n, Hkv, H // Hkv, Dh).transpose(0, 1).reshape(Hkv, n * (H // Hkv), Dh)


def _plain_sparse(s):
    c = s.case
    H, Hkv, Dh, block = (c[k] for k in ("H", "Hkv", "Dh", "block"))
    G = H // Hkv
    for b in range(c["B"]):
        m, L = int(s.rows[b]), int(s.L[b])
        n_blk = -(-L // block)
        take = min(c["sel"], n_blk)
        # the score of a block, summed over the heads that share its keys, in 64 bits: near scores keep their order
        qs = s.q[b, :m].double().view(m, Hkv, G, Dh).sum(2).transpose(0, 1).contiguous()
        score = torch.matmul(qs, s.means[b, :, :n_blk].double().transpose(1, 2).contiguous())
        score[:, :, max(0, n_blk - LAST):] = math.inf
        score[:, :, :FIRST] = math.inf
        best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :take]
        s.sel[b, :m, :, :take] = best.sort(-1).values.transpose(0, 1).int()
        chosen = torch.zeros(Hkv, m, n_blk, dtype=torch.bool, device="cuda").scatter_(2, best, True)
        see = torch.cat([chosen.repeat_interleave(block, 2)[:, :, :L],
                         s.paths[b][:m, :m].expand(Hkv, m, m)], -1).repeat_interleave(G, 1)
        p = _softmax_parts(_row_heads(s.q[b, :m].float(), Hkv), s.kc[b, :, : L + m].float(), see, 1 / math.sqrt(Dh))
        o = torch.matmul(p, s.vc[b, :, : L + m].float())
        s.out[b, :m] = o.view(Hkv, m, G, Dh).transpose(0, 1).reshape(m, H, Dh).to(s.out.dtype)
    return {"out": s.out, "blocks": s.sel}


def _plain_weights(s):
    c = s.case
    H, Hkv, Dh = (c[k] for k in ("H", "Hkv", "Dh"))
    G = H // Hkv
    for b in range(c["B"]):
        m, L = int(s.rows[b]), int(s.L[b])
        see = torch.ones(m, L + m, dtype=torch.bool, device="cuda")
        see[:, L:] = s.paths[b][:m, :m]
        p = _softmax_parts(_row_heads(s.q[b, :m].float(), Hkv), s.kc[b, :, : L + m].float(),
                           see.repeat_interleave(G, 0)[None], 1 / math.sqrt(Dh))
        o = torch.matmul(p, s.vc[b, :, : L + m].float())
        s.out[b, :m] = o.view(Hkv, m, G, Dh).transpose(0, 1).reshape(m, H, Dh).to(s.out.dtype)
        if s.rating is not None:
            p = p * s.rating[b, :m].repeat_interleave(G)[None, :, None]
        got = p.sum(1)
        got[:, :L] += c["decay"] * s.w[b, :, :L]      # the tree's own slots are new: no earlier weight
        s.wo[b, :, : L + m] = got
    return {"out": s.out, "weights": s.wo}


def _plain_evict(s):
    c = s.case
    for b in range(c["B"]):
        L = int(s.L[b])
        keep = min(L, c["budget"])
        if L <= c["budget"]:
            kept = torch.arange(L, device="cuda").expand(c["slices"], L)
        else:
            w = s.w[b, :, :L].clone()
            w[:, : c["first"]] = math.inf
            w[:, L - c["last"]:] = math.inf
            kept = torch.sort(w, dim=-1, descending=True, stable=True).indices[:, :keep].sort(-1).values
        at = kept[..., None].expand(-1, -1, c["Dh"])
        s.ko[b, :, :keep] = torch.gather(s.kc[b], 1, at)
        s.vo[b, :, :keep] = torch.gather(s.vc[b], 1, at)
        s.wo[b, :, :keep] = torch.gather(s.w[b], 1, kept)
        s.kept[b, :, :keep] = kept.int()
        s.new_len[b] = keep
    return {"k": s.ko, "v": s.vo, "weights": s.wo, "kept": s.kept, "length": s.new_len}


PLAIN = {"rope": _plain_rope, "keys": _plain_keys, "sparse": _plain_sparse, "weights": _plain_weights,
         "evict": _plain_evict}


# ------------------------------------------------------------------------------ what it takes
def _rows(c):
    n = c["n"]
    return c["B"] * n if not c["ragged"] or c["B"] == 1 else n + (c["B"] - 1) * (max(1, n // 4) + n) / 2


def _slots(c):
    return c["hi"] + (c["B"] - 1) * (c["lo"] + c["hi"]) / 2


def work(case):
    kind, es, B, Dh = case["kind"], _esize(case), case["B"], case["Dh"]
    L = _slots(case)
    if kind == "rope":
        rows = _rows(case)
        vals = rows * (case["H"] + 2 * case["Hkv"]) * Dh
        turned = rows * (case["H"] + case["Hkv"]) * case["rot"]
        return {"bytes": 2 * es * vals + 4 * rows, "flops": 3 * turned}
    if kind == "keys":
        if case["last"]:
            L = B * (case["last"] + case["block"] / 2)
        vals = L * case["Hkv"] * Dh
        return {"bytes": es * vals + 4 * vals / case["block"], "flops": vals}
    if kind == "evict":
        keep = B * min(case["budget"], L / B)
        moved = keep * case["slices"]
        return {"bytes": 4 * es * moved * Dh + 4 * L * case["slices"] + 8 * moved, "flops": L * case["slices"]}
    rows, H, Hkv = _rows(case), case["H"], case["Hkv"]
    ends = 2 * es * rows * H * Dh + 16 * rows
    tail = 2 * es * rows * Hkv * Dh
    if kind == "weights":
        return {"bytes": ends + tail + 2 * es * L * Hkv * Dh + 8 * L * Hkv,
                "flops": rows * H * (L / B + rows / B / 2) * (4 * Dh + 1)}
    # every row takes `sel` blocks; what different rows add is not counted as read twice
    blocks = L / case["block"]
    seen = min(case["sel"] * case["block"], L / B)
    return {"bytes": ends + tail + 4 * blocks * Hkv * Dh + 2 * es * B * seen * Hkv * Dh + 4 * rows * Hkv * case["sel"],
            "flops": 2 * rows * Hkv * blocks / B * Dh + 4 * rows * H * (seen + rows / B / 2) * Dh}


# ------------------------------------------------------------------------------ in 64 bits
def _exact_rope(s):
    c = s.case
    rot, half = c["rot"], c["rot"] // 2
    freq = []
    base = THETA * c["factor"] ** (rot / (rot - 2.0)) if c["scaling"] == "base" and rot > 2 else THETA
    for i in range(half):
        f = math.exp(-2.0 * i / rot * math.log(base))
        if c["scaling"] == "linear":
            f /= c["factor"]
        if c["scaling"] == "ramp":
            edge = [rot * math.log(c["orig"] / (turns * 2 * math.pi)) / (2 * math.log(THETA)) for turns in (FAST, SLOW)]
            lo, hi = max(0, math.floor(edge[0])), min(rot - 1, math.ceil(edge[1]))
            t = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            f = (1.0 - t) * f + t * f / c["factor"]
        freq.append(f)
    gain = 1.0 + 0.1 * math.log(c["factor"]) if c["scaling"] == "ramp" else 1.0
    e = torch.polar(torch.full((half,), gain, dtype=torch.float64, device="cuda"),
                    s.pos.double()[..., None] * torch.tensor(freq, dtype=torch.float64, device="cuda"))[:, :, None]

    def turned(x):
        x = x.double().clone()
        first, second = (slice(0, half), slice(half, rot)) if c["layout"] == HALF else (slice(0, rot, 2), slice(1, rot, 2))
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * e
        x[..., first], x[..., second] = z.real, z.imag
        return x

    q, k, v = turned(s.q), turned(s.k), s.v.double()
    out, kc, vc = s.out.double(), s.kc.double(), s.vc.double()
    for b in range(c["B"]):
        m, L = int(s.rows[b]), int(s.L[b])
        out[b, :m] = q[b, :m]
        kc[b, :, L: L + m] = k[b, :m].transpose(0, 1)
        vc[b, :, L: L + m] = v[b, :m].transpose(0, 1)
    return {"q": out, "k_cache": kc, "v_cache": vc}


def _exact_keys(s):
    c, out = s.case, s.out.double()
    for b in range(c["B"]):
        L = int(s.L[b])
        slot = torch.arange(L, device="cuda")
        blk = slot // c["block"]
        n_blk = int(blk[-1]) + 1
        total = torch.zeros(c["Hkv"], n_blk, c["Dh"], dtype=torch.float64, device="cuda")
        total.index_add_(1, blk, s.kc[b, :, :L].double())
        j0 = (L - c["last"]) // c["block"] if c["last"] else 0
        out[b, :, j0:n_blk] = (total / torch.bincount(blk)[None, :, None])[:, j0:]
    return out


def _exact_attend(q, k, v, see, scale):
    """One head: q [r][Dh], k and v [t][Dh], see [r][t] -> outputs and weights."""
    x = (q @ k.t().contiguous() * scale).masked_fill(~see, -math.inf)
    p = torch.nan_to_num(torch.exp(x - torch.logsumexp(x, 1, keepdim=True)), nan=0.0)
    return p @ v, p


def _exact_sparse(s):
    c = s.case
    Hkv, Dh, block = (c[k] for k in ("Hkv", "Dh", "block"))
    G = c["H"] // Hkv
    out, sel = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda"), s.sel.clone()
    for b in range(c["B"]):
        m, L = int(s.rows[b]), int(s.L[b])
        n_blk = (L + block - 1) // block
        take = min(n_blk, c["sel"])
        j = torch.arange(n_blk, device="cuda")
        fixed = (j < FIRST) | (j >= n_blk - LAST)
        block_of = torch.arange(L, device="cuda") // block
        tail = torch.from_numpy(s.path[b][:m, :m]).cuda()
        for h in range(Hkv):
            q = s.q[b, :m, h * G: (h + 1) * G].double()
            score = (q[:, :, None] * s.means[b, h, :n_blk].double()).sum((1, 3)) if m * G * n_blk * Dh < 2 ** 26 else \
                torch.stack([(q[i].sum(0) * s.means[b, h, :n_blk].double()).sum(1) for i in range(m)])
            score = score.masked_fill(fixed, math.inf)
            # a block's rank: how many score more, or as much at a lower index
            rank = torch.stack([((r[None] > r[:, None]) | ((r[None] == r[:, None]) & (j[None] < j[:, None]))).sum(1)
                                for r in score])
            chosen = rank < take
            sel[b, :m, h, :take] = chosen.nonzero()[:, 1].view(m, take).int()
            see = torch.cat([chosen[:, block_of], tail], 1)
            for u in range(G):
                out[b, :m, h * G + u] = _exact_attend(q[:, u].contiguous(), s.kc[b, h, : L + m].double(),
                                                      s.vc[b, h, : L + m].double(), see, Dh ** -0.5)[0]
    return {"out": out, "blocks": sel}


def _exact_weights(s):
    c = s.case
    Hkv, Dh = c["Hkv"], c["Dh"]
    G = c["H"] // Hkv
    out, wo = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda"), s.wo.double()
    for b in range(c["B"]):
        m, L = int(s.rows[b]), int(s.L[b])
        see = torch.cat([torch.ones(m, L, dtype=torch.bool), torch.from_numpy(s.path[b][:m, :m])], 1).cuda()
        rating = torch.ones(m, dtype=torch.float64, device="cuda") if s.rating is None else s.rating[b, :m].double()
        for h in range(Hkv):
            wo[b, h, :L] = c["decay"] * s.w[b, h, :L].double()
            for u in range(G):
                o, p = _exact_attend(s.q[b, :m, h * G + u].double(), s.kc[b, h, : L + m].double(),
                                     s.vc[b, h, : L + m].double(), see, Dh ** -0.5)
                out[b, :m, h * G + u] = o
                wo[b, h, : L + m] += rating @ p
    return {"out": out, "weights": wo}


def _exact_evict(s):
    c = s.case
    ko, vo, wo, kept = s.ko.double(), s.vo.double(), s.wo.double(), s.kept.clone()
    w = s.w.cpu().numpy()
    for b in range(c["B"]):
        L = int(s.L[b])
        keep = min(c["budget"], L)
        for h in range(c["slices"]):
            at = np.arange(L)
            if L > keep:
                mid = np.arange(c["first"], L - c["last"])
                order = np.lexsort((mid, -w[b, h, mid]))[: keep - c["first"] - c["last"]]
                at = np.concatenate([at[: c["first"]], np.sort(mid[order]), at[L - c["last"]:]])
            at = torch.from_numpy(at).cuda()
            ko[b, h, :keep], vo[b, h, :keep] = s.kc[b, h, at].double(), s.vc[b, h, at].double()
            wo[b, h, :keep] = s.w[b, h, at].double()
            kept[b, h, :keep] = at.int()
    return {"k": ko, "v": vo, "weights": wo, "kept": kept, "length": _dev(np.minimum(s.L, c["budget"]))}


def exact(case, seed):
    s = _inputs(case, seed)
    return {"rope": _exact_rope, "keys": _exact_keys, "sparse": _exact_sparse, "weights": _exact_weights,
            "evict": _exact_evict}[case["kind"]](s)


if __name__ == "__main__":
    for c in listed() + [draw(random.Random(i)) for i in range(4)]:
        print(c, work(c))
