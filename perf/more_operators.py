"""Operators of caches in eight bits and of caches that a batch shares, as measured workloads.

A case is one pass through the public entry points of `paper_2512_21857_amd.runtime` (`own`
true), or the same operators in elementary torch operations (`own` false).  The operators belong
together: queries and keys are normalised and rotated head by head as keys and values are appended to
a cache, which may hold them in eight bits with a scale for each row; caches are turned from one type
into another and read back; tree attention reads such a cache, and a prefix that a batch of sequences
shares once for all of them; an accepted path is moved up in it.

Kinds
  append   norms of queries and keys, rotation, append to a cache of any type; rows of an eight-bit
           cache are read back
  convert  slots of an eight-bit cache read back, or a plain cache's slots put in eight bits and read back
  compact  an accepted path moved to the end of the prefix, in an eight-bit cache, and read back
  attn     tree attention over a cache of any type, behind a prefix of its own or one shared by a group

Shapes are those of this repository's configurations (20 heads of 64 in 36 layers; 32 heads of 128 in
32 layers; the tiny fp32 model's 4 heads of 64; trees of up to 61 and 128 rows, 2352-token images) and
generic long-context ones with grouped heads (32 query heads over 8 key-value heads, up to 65536 slots).
"""
import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

HALF, INTERLEAVED = "half", "interleaved"
EPS, THETA = 1e-5, 10000.0


def listed():
    return [
        # one image's 61-row tree in one layer of a model with query and key norms: latency
        dict(name="append_tree_61", kind="append", B=1, n=61, H=32, Hkv=32, Dh=128, rot=128, layout=HALF, norm="shared",
             type="e4m3", dtype="bf16", lo=2300, hi=2300, cap=2560, ragged=False),
        # a long prompt of a grouped-head model, a gain for every head, half of each head rotated in neighbouring pairs
        dict(name="append_prompt_4001", kind="append", B=1, n=4001, H=32, Hkv=8, Dh=128, rot=64, layout=INTERLEAVED,
             norm="heads", type="int8", dtype="bf16", lo=17, hi=17, cap=4096, ragged=False),
        # sixteen caches read back, as before a call that takes plain caches only
        dict(name="convert_read_16x4k", kind="convert", B=16, Hkv=8, Dh=128, lo=512, hi=4096, cap=4160, type="e4m3",
             dtype="bf16", write=False),
        # a prefilled prompt put in eight bits, one layer
        dict(name="convert_prompt_1100", kind="convert", B=1, Hkv=32, Dh=128, lo=1100, hi=1100, cap=1216, type="int8",
             dtype="bf16", write=True),
        # the accepted path of one image in all slices of a 32-layer model
        dict(name="compact_image", kind="compact", B=1, Hkv=1024, Dh=128, n=61, a=12, lo=2300, hi=2300, cap=2432,
             type="e4m3", dtype="bf16"),
        # of four images, 36 layers of 20 heads of 64
        dict(name="compact_batch_4", kind="compact", B=4, Hkv=720, Dh=64, n=61, a=5, lo=100, hi=600, cap=768, type="int8",
             dtype="bf16"),
        # a 17-row tree early in an image: latency of a launch or two
        dict(name="attn_tree_17", kind="attn", B=1, n=17, H=20, Hkv=20, Dh=64, groups=0, plo=0, phi=0, pcap=0, lo=300,
             hi=300, cap=448, type="e4m3", dtype="bf16", ragged=False),
        # one token of one long sequence
        dict(name="attn_decode_64k", kind="attn", B=1, n=1, H=32, Hkv=8, Dh=128, groups=0, plo=0, phi=0, pcap=0, lo=65333,
             hi=65333, cap=65536, type="int8", dtype="bf16", ragged=False),
        # the ragged trees of sixteen images somewhere in theirs
        dict(name="attn_16x61", kind="attn", B=16, n=61, H=32, Hkv=32, Dh=128, groups=0, plo=0, phi=0, pcap=0, lo=512,
             hi=2400, cap=2560, type="e4m3", dtype="bf16", ragged=True),
        # the fp32 model, two prompts with two images each
        dict(name="prefix_tiny_2x2", kind="attn", B=4, n=17, H=4, Hkv=4, Dh=64, groups=2, plo=150, phi=200, pcap=256,
             lo=20, hi=100, cap=192, type="f32", dtype="f32", ragged=True),
        # sixteen images behind one long prompt, near the end of their first rows: many rows for each key
        dict(name="prefix_images_16x61", kind="attn", B=16, n=61, H=32, Hkv=32, Dh=128, groups=1, plo=2100, phi=2100,
             pcap=2112, lo=64, hi=576, cap=704, type="bf16", dtype="bf16", ragged=True),
        # one token of each of 64 sequences behind a very long prefix in eight bits, grouped heads
        dict(name="prefix_decode_64x1", kind="attn", B=64, n=1, H=32, Hkv=8, Dh=128, groups=1, plo=32700, phi=32700,
             pcap=32768, lo=1, hi=512, cap=576, type="int8", dtype="bf16", ragged=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(32, 32, 128), (20, 20, 64), (4, 4, 64), (32, 8, 128), (16, 2, 128), (24, 8, 64), (8, 1, 64)]


def _draw(rng):
    kind = rng.choice(["append", "append", "convert", "compact", "attn", "attn", "attn", "attn"])
    H, Hkv, Dh = rng.choice(HEADS)
    B = rng.choice([1, 1, 1, 2, 3, 7, 16])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    eight = rng.choice(["e4m3", "int8"])
    if kind == "append":
        Dh = rng.choice([Dh, Dh, 96])
        n, lo = _log_int(rng, 1, 4096), _log_int(rng, 1, 4096)
        return dict(kind=kind, B=B, n=n, H=H, Hkv=Hkv, Dh=Dh, rot=rng.choice([Dh, Dh, Dh // 2, 2 * rng.randint(1, Dh // 2)]),
                    layout=rng.choice([HALF, INTERLEAVED]), norm=rng.choice(["shared", "shared", "heads", "none"]),
                    type=rng.choice([eight, eight, dtype]), dtype=dtype, lo=lo, hi=lo + rng.randint(0, 600),
                    cap=lo + n + 600, ragged=rng.random() < 0.5)
    if kind == "convert":
        lo = _log_int(rng, 1, 32768)
        hi = lo if B == 1 else rng.randint(lo, 32768)
        return dict(kind=kind, B=B, Hkv=Hkv, Dh=rng.choice([Dh, Dh, 96]), lo=lo, hi=hi, cap=hi + rng.randint(0, 300),
                    type=eight, dtype=dtype, write=rng.random() < 0.5)
    if kind == "compact":
        n = rng.randint(12, 128)
        lo = _log_int(rng, 1, 2300)
        hi = rng.randint(lo, 2300)
        return dict(kind=kind, B=B, Hkv=Hkv * rng.choice([1, 8, 32]), Dh=Dh, n=n, a=rng.randint(1, (n - 1) // 2), lo=lo,
                    hi=hi, cap=hi + n + rng.randint(0, 200), type=eight, dtype=dtype)
    kind_of = rng.choice([eight, eight, "bf16", "f32"])
    dtype = "f32" if kind_of == "f32" else "bf16"
    groups = rng.choice([0, 1, 1, 2]) if kind_of in ("e4m3", "int8") else rng.choice([1, 1, 2])
    B = rng.choice([2, 4, 8, 16, 64]) if groups else B
    n = _log_int(rng, 1, 128)
    lo = _log_int(rng, 1, 2400 if groups else 32000)
    hi = rng.randint(lo, 2400 if groups else 32000)
    plo = _log_int(rng, 40, 32000) if groups else 0
    phi = plo + rng.randint(0, plo // 4) if groups > 1 else plo
    return dict(kind=kind, B=B, n=n, H=H, Hkv=Hkv, Dh=Dh, groups=groups, plo=plo, phi=phi,
                pcap=phi + rng.randint(0, 100) if groups else 0, lo=lo, hi=hi, cap=hi + n + rng.randint(0, 300),
                type=kind_of, dtype=dtype, ragged=rng.random() < 0.5)


def draw(rng):
    """A case of the listed ones' ranges that costs no more than the largest listed one of its kind."""
    most = {}
    for c in listed():
        w = work(c)
        most[c["kind"]] = [max(a, w[k]) for a, k in zip(most.get(c["kind"], [0, 0]), ("bytes", "flops"))]
    while True:
        c = _draw(rng)
        w = work(c)
        size = c["B"] * c["Hkv"] * c["cap"] * c["Dh"] + c.get("groups", 0) * c["Hkv"] * c.get("pcap", 0) * c["Dh"]
        scores = c["B"] * c["n"] * c["H"] * (c["cap"] + c["pcap"]) if c["kind"] == "attn" else 0
        if w["bytes"] <= most[c["kind"]][0] and w["flops"] <= most[c["kind"]][1] and size <= 3.5e8 and scores <= 1.5e8:
            return c


# ------------------------------------------------------------------------------ inputs
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
TOP = {"int8": 127.0, "e4m3": 448.0}      # the largest value of each eight-bit type


def _gen(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000 + tag)
    return g


def _dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def _normal(g, dt, *shape):
    return torch.empty(*shape, dtype=dt, device="cuda").normal_(generator=g)


def _quantised(x, kind):
    """Rows x [..., Dh] in eight bits: codes and a scale for each row, the row's largest size being the
    type's.  The quotient is rounded to 32 bits, then to the type."""
    y = x.double()
    scale = (y.abs().amax(-1).float().double() / TOP[kind]).float()
    by = torch.where(scale > 0, scale, torch.ones_like(scale)).double()[..., None]
    t = (y / by).float().clamp(-TOP[kind], TOP[kind])
    return (t.round() if kind == "int8" else t).to(TORCH[kind]), scale


def _values(codes, scale, dt):
    return (codes.float() * scale[..., None]).to(dt)


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


def _lengths(rng, lo, hi, count):
    L = rng.integers(lo, hi + 1, size=count)
    L[0] = hi
    return L.astype(np.int32)


def _filled(g, kind, *shape):
    """A cache of that type with keys and values as a model makes them: neighbouring keys have much in
    common, and a few dims of the keys are much larger than the others."""
    B, heads, cap, Dh = shape
    dt = TORCH[kind] if kind in ("f32", "bf16") else torch.bfloat16
    k, v = _normal(g, dt, *shape), _normal(g, dt, *shape)
    whole = cap // 32 * 32
    k[:, :, :whole].view(B, heads, whole // 32, 32, Dh).add_(0.7 * _normal(g, dt, B, heads, whole // 32, 1, Dh))
    k[..., ::31] *= 3.0
    if kind in ("f32", "bf16"):
        return [k, v, None, None]
    (kc, ks), (vc, vs) = _by_parts(k, kind), _by_parts(v, kind)
    return [kc, vc, ks, vs]


def _by_parts(x, kind):
    """_quantised, some heads at a time: its 64-bit values take four times the memory."""
    at = max(1, 2 ** 26 // max(1, x[:, :1].numel()))
    parts = [_quantised(x[:, i: i + at], kind) for i in range(0, x.shape[1], at)]
    return torch.cat([p[0].view(torch.int8) for p in parts], 1).view(TORCH[kind]), torch.cat([p[1] for p in parts], 1)


def _random_codes(g, kind, *shape):
    """Codes and scales of a cache whose values no one adds up: uniform codes, none of them NaN (of e4m3, the
    bytes 127 and -1)."""
    c = torch.randint(-126, 127, shape, dtype=torch.int8, device="cuda", generator=g)
    c.masked_fill_(c == -1, 1)
    return c.view(TORCH[kind]), torch.rand(shape[:-1], device="cuda", generator=g) + 0.01


def _plain_window(case, slots):
    """Where values are read back to: two plain caches [B][Hkv][slots][Dh] of zeros."""
    return [torch.zeros(case["B"], case["Hkv"], slots, case["Dh"], dtype=TORCH[case["dtype"]], device="cuda")
            for _ in range(2)]


def _inputs(case, seed):
    """What a user's program has in hand, apart from handles and workspaces."""
    kind, B, Hkv, Dh, cap, dt = case["kind"], case["B"], case["Hkv"], case["Dh"], case["cap"], TORCH[case["dtype"]]
    rng, g = np.random.default_rng([int(seed), 17]), _gen(seed, 18)
    s = SimpleNamespace(case=case, L=_lengths(rng, case["lo"], case["hi"], B))
    s.kv_len = _dev(s.L)
    if kind == "append":
        n, H = case["n"], case["H"]
        s.rows, parent = _trees(dict(case, n=min(n, 128)), rng)
        s.rows = np.maximum(1, s.rows * n // min(n, 128)).astype(np.int32)
        s.n_rows = _dev(s.rows)
        # a tree's rows share positions by depth, a prompt's follow one another
        depth = np.tile(np.arange(n, dtype=np.int32), (B, 1)) if n > 128 else np.zeros((B, n), dtype=np.int32)
        if n <= 128:
            for b in range(B):
                for i in range(1, n):
                    depth[b, i] = depth[b, parent[b, i]] + 1 if parent[b, i] >= 0 else 0
        s.pos = _dev(s.L[:, None] + depth)
        # the three parts of one projection's output rows
        qkv = 2.0 * _normal(g, dt, B, n, (H + 2 * Hkv) * Dh)
        s.q = qkv[..., : H * Dh].unflatten(-1, (H, Dh))
        s.k = qkv[..., H * Dh: (H + Hkv) * Dh].unflatten(-1, (Hkv, Dh))
        s.v = qkv[..., (H + Hkv) * Dh:].unflatten(-1, (Hkv, Dh))
        s.q_norm = s.k_norm = None
        if case["norm"] != "none":
            s.q_norm, s.k_norm = (1.0 + 0.2 * _normal(g, torch.float32, *([h] if case["norm"] == "heads" else []), Dh)
                                  for h in (H, Hkv))
        s.out = torch.zeros(B, n, H, Dh, dtype=dt, device="cuda")
        if case["type"] in TOP:
            (s.kc, s.ks), (s.vc, s.vs) = (_random_codes(g, case["type"], B, Hkv, cap, Dh) for _ in range(2))
            s.kw, s.vw = _plain_window(case, n)
        else:
            s.kc, s.vc, s.ks, s.vs = _filled(g, case["type"], B, Hkv, cap, Dh)
        return s
    if kind == "convert":
        if case["write"]:
            s.k0, s.v0 = (_normal(g, dt, B, Hkv, cap, Dh) for _ in range(2))     # the plain cache
            (s.kc, s.ks), (s.vc, s.vs) = (_random_codes(g, case["type"], B, Hkv, cap, Dh) for _ in range(2))
        else:
            (s.kc, s.ks), (s.vc, s.vs) = (_random_codes(g, case["type"], B, Hkv, cap, Dh) for _ in range(2))
        s.kw, s.vw = _plain_window(case, cap)
        return s
    if kind == "compact":
        n, a = case["n"], case["a"]
        (s.kc, s.ks), (s.vc, s.vs) = (_random_codes(g, case["type"], B, Hkv, cap, Dh) for _ in range(2))
        # a path's nodes lie past the first levels' (indices a + 1 and more), in rising order
        s.n_acc = rng.integers(max(1, a // 2), a + 1, size=B).astype(np.int32)
        s.n_acc[0] = a
        s.path = np.zeros((B, a + 1), dtype=np.int32)
        for b in range(B):
            s.path[b, 1:] = np.sort(rng.choice(np.arange(a + 1, n), size=a, replace=False))
        s.acc, s.node, s.first = _dev(s.n_acc), _dev(s.path), _dev(s.L + 1)
        s.kw, s.vw = _plain_window(case, a)
        return s
    n, H = case["n"], case["H"]
    s.kc, s.vc, s.ks, s.vs = _filled(g, case["type"], B, Hkv, cap, Dh)
    # the rows of one tree ask for much the same
    s.q = (_normal(g, torch.float32, B, 1, H, Dh) + 0.5 * _normal(g, torch.float32, B, n, H, Dh)).to(dt)
    s.rows, parent = _trees(case, rng)
    s.path = np.stack([_path(parent[b], s.rows[b], n) for b in range(B)])
    s.mask = _dev(np.stack([_words(p) for p in s.path]), np.int64)
    s.n_rows = _dev(s.rows)
    s.out = torch.zeros(B, n, H, Dh, dtype=dt, device="cuda")
    if case["groups"]:
        s.P = _lengths(rng, case["plo"], case["phi"], case["groups"])
        s.prefix_len = _dev(s.P)
        s.pk, s.pv, s.pks, s.pvs = _filled(g, case["type"], case["groups"], Hkv, case["pcap"], Dh)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        s.paths = _dev(s.path, bool) if case["kind"] == "attn" else None
        return s
    from paper_2512_21857_amd import runtime as rt
    s.cache = rt.KVCache(s.kc, s.vc, s.ks, s.vs)
    if case["kind"] == "append":
        s.freq, s.gain = rt.rope_freqs(case["rot"], THETA)
    if hasattr(s, "kw"):
        s.window = rt.KVCache(s.kw, s.vw)
    if case["kind"] == "convert" and case["write"]:
        s.source = rt.KVCache(s.k0, s.v0)
    if case["kind"] == "attn":
        s.prefix = rt.KVCache(s.pk, s.pv, s.pks, s.pvs) if case["groups"] else None
        s.ws = rt.cache_tree_attn_workspace(case["H"], case["n"], s.cache, prefix=s.prefix)
    return s


# ------------------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else PLAIN[s.case["kind"]](s)


def _run_own(s):
    from paper_2512_21857_amd import runtime as rt
    c = s.case
    if c["kind"] == "append":
        rt.norm_rope_append(s.q, s.k, s.v, s.pos, s.kv_len, s.n_rows, s.freq, s.cache, q_norm=s.q_norm, k_norm=s.k_norm,
                            eps=EPS, layout=c["layout"], gain=s.gain, out=s.out)
        if c["type"] not in TOP:
            return {"q": s.out, "k": s.kc, "v": s.vc}
        rt.cache_convert(s.cache, s.window, s.n_rows, n_max=c["n"], src_start=s.kv_len)
        return {"q": s.out, "k": s.kw, "v": s.vw}
    if c["kind"] == "convert":
        if c["write"]:
            rt.cache_convert(s.source, s.cache, s.kv_len)
        rt.cache_convert(s.cache, s.window, s.kv_len)
        return {"k": s.kw, "v": s.vw}
    if c["kind"] == "compact":
        rt.cache_compact(s.cache, s.kv_len, s.node, s.acc, c["a"])
        rt.cache_convert(s.cache, s.window, s.acc, n_max=c["a"], src_start=s.first)
        return {"k": s.kw, "v": s.vw}
    if c["groups"]:
        return rt.cache_tree_attn(s.q, s.cache, s.kv_len, s.n_rows, s.n_rows, s.mask, prefix=s.prefix,
                                  prefix_len=s.prefix_len, out=s.out, workspace=s.ws)
    return rt.cache_tree_attn(s.q, s.cache, s.kv_len, s.n_rows, s.n_rows, s.mask, out=s.out, workspace=s.ws)


# ------------------------------------------------------------------------------ plain forms
def _rows_of(lengths, n):
    """(sequence, row) of every row i < lengths[b]."""
    return (torch.arange(n, device="cuda")[None] < lengths[:, None]).nonzero(as_tuple=True)


def _plain_append(s):
    c, rot = s.case, s.case["rot"]
    # in 64 bits up to the rounding: a quotient next to a border between two codes decides by its last digits
    angle = s.pos.double()[..., None] * THETA ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / rot)
    cos, sin = torch.cos(angle)[:, :, None], torch.sin(angle)[:, :, None]

    def made(x, weight):
        y = x.double()
        if weight is not None:
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS) * weight.double()
        if c["layout"] == HALF:
            a, b = y[..., : rot // 2], y[..., rot // 2: rot]
            t = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        else:
            a, b = y[..., 0:rot:2], y[..., 1:rot:2]
            t = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        return torch.cat([t, y[..., rot:]], -1)

    b, i = _rows_of(s.n_rows, c["n"])
    slot = s.kv_len.long()[b] + i
    s.out[b, i] = made(s.q, s.q_norm)[b, i].to(s.out.dtype)
    k, v = made(s.k, s.k_norm)[b, i], s.v[b, i]
    if c["type"] not in TOP:
        s.kc[b, :, slot], s.vc[b, :, slot] = k.to(s.kc.dtype), v
        return {"q": s.out, "k": s.kc, "v": s.vc}
    kc, ks = _quantised(k, c["type"])
    vc, vs = _quantised(v, c["type"])
    s.kc.view(torch.int8)[b, :, slot], s.vc.view(torch.int8)[b, :, slot] = kc.view(torch.int8), vc.view(torch.int8)
    s.ks[b, :, slot], s.vs[b, :, slot] = ks, vs
    s.kw[b, :, i] = _values(_codes(s.kc, c)[b, :, slot], s.ks[b, :, slot], s.kw.dtype)
    s.vw[b, :, i] = _values(_codes(s.vc, c)[b, :, slot], s.vs[b, :, slot], s.vw.dtype)
    return {"q": s.out, "k": s.kw, "v": s.vw}


class _codes:
    """Rows of a cache of codes, which torch indexes as bytes."""

    def __init__(self, x, c):
        self.x, self.kind = x.view(torch.int8), TORCH[c["type"]]

    def __getitem__(self, at):
        return self.x[at].contiguous().view(self.kind)


def _plain_convert(s):
    c = s.case
    b, i = _rows_of(s.kv_len, c["cap"])
    if c["write"]:
        for plain, codes, scale in ((s.k0, s.kc, s.ks), (s.v0, s.vc, s.vs)):
            x, by = _quantised(plain[b, :, i], c["type"])
            codes.view(torch.int8)[b, :, i], scale[b, :, i] = x.view(torch.int8), by
    s.kw[b, :, i] = _values(_codes(s.kc, c)[b, :, i], s.ks[b, :, i], s.kw.dtype)
    s.vw[b, :, i] = _values(_codes(s.vc, c)[b, :, i], s.vs[b, :, i], s.vw.dtype)
    return {"k": s.kw, "v": s.vw}


def _plain_compact(s):
    c = s.case
    b, m = _rows_of(s.acc, c["a"])
    to = s.kv_len.long()[b] + 1 + m
    frm = s.kv_len.long()[b] + s.node.long()[b, 1 + m]
    for codes, scale, window in ((s.kc.view(torch.int8), s.ks, s.kw), (s.vc.view(torch.int8), s.vs, s.vw)):
        codes[b, :, to], scale[b, :, to] = codes[b, :, frm], scale[b, :, frm]
        window[b, :, m] = _values(_codes(codes, c)[b, :, to], scale[b, :, to], window.dtype)
    return {"k": s.kw, "v": s.vw}


def _cache_values(x, scale):
    return x.float() if scale is None else x.float() * scale[..., None]


def _plain_attn(s):
    c = s.case
    B, n, H, Hkv, Dh, cap = (c[k] for k in ("B", "n", "H", "Hkv", "Dh", "cap"))
    G, groups, scale = H // Hkv, c["groups"], 1 / math.sqrt(Dh)
    rows = s.q.float().view(B, n, Hkv, G, Dh).transpose(1, 2).reshape(B, Hkv, n * G, Dh)
    # what each row sees of its own cache: the slots before the tree, and of the tree its path
    at = torch.arange(cap, device="cuda")[None] - s.kv_len[:, None]
    tail = (at >= 0) & (at < n)
    see = torch.gather(s.paths, 2, at.clamp(0, n - 1)[:, None].expand(B, n, cap).long()) & tail[:, None] | (at < 0)[:, None]
    see = see.repeat_interleave(G, 1)[:, None]
    x = torch.matmul(rows, _cache_values(s.kc, s.ks).transpose(2, 3).contiguous()) * scale
    x = x.masked_fill_(~see, -math.inf)
    if groups:
        # every row of a group against the group's prefix
        many = rows.view(groups, B // groups, Hkv, n * G, Dh).transpose(1, 2).reshape(groups, Hkv, -1, Dh)
        y = torch.matmul(many, _cache_values(s.pk, s.pks).transpose(2, 3).contiguous()) * scale
        behind = torch.arange(c["pcap"], device="cuda")[None] >= s.prefix_len[:, None]
        y = y.masked_fill_(behind[:, None, None], -math.inf)
        y = y.view(groups, Hkv, B // groups, n * G, c["pcap"]).transpose(1, 2).reshape(B, Hkv, n * G, c["pcap"])
        top = torch.maximum(x.amax(-1, keepdim=True), y.amax(-1, keepdim=True))
        ex, ey = torch.exp(x - top), torch.exp(y - top)
        total = ex.sum(-1, keepdim=True) + ey.sum(-1, keepdim=True)
        ey = ey.view(groups, B // groups, Hkv, n * G, c["pcap"]).transpose(1, 2).reshape(groups, Hkv, -1, c["pcap"])
        o = torch.matmul(ey, _cache_values(s.pv, s.pvs)).view(groups, Hkv, B // groups, n * G, Dh)
        o = o.transpose(1, 2).reshape(B, Hkv, n * G, Dh) + torch.matmul(ex, _cache_values(s.vc, s.vs))
    else:
        ex = torch.exp(x - x.amax(-1, keepdim=True))
        total = ex.sum(-1, keepdim=True)
        o = torch.matmul(ex, _cache_values(s.vc, s.vs))
    o = (o / total).view(B, Hkv, n, G, Dh).transpose(1, 2).reshape(B, n, H, Dh)
    b, i = _rows_of(s.n_rows, n)
    s.out[b, i] = o[b, i].to(s.out.dtype)
    return s.out


PLAIN = {"append": _plain_append, "convert": _plain_convert, "compact": _plain_compact, "attn": _plain_attn}


# ------------------------------------------------------------------------------ what it takes
ESIZE = {"f32": 4, "bf16": 2, "int8": 1, "e4m3": 1}


def _row_bytes(case):
    """Bytes of one slot of one head, keys and values."""
    return 2 * (case["Dh"] * ESIZE[case["type"]] + (4 if case["type"] in TOP else 0))


def _rows(c):
    n = c["n"]
    return c["B"] * n if not c["ragged"] or c["B"] == 1 else n + (c["B"] - 1) * (max(1, n // 4) + n) / 2


def _slots(c):
    return c["hi"] + (c["B"] - 1) * (c["lo"] + c["hi"]) / 2


def work(case):
    kind, es, B, Hkv, Dh = case["kind"], ESIZE[case["dtype"]], case["B"], case["Hkv"], case["Dh"]
    plain = 2 * Hkv * Dh * es            # one row's keys and values in the rows' type
    back = plain if case["type"] in TOP else 0
    if kind == "append":
        rows = _rows(case)
        return {"bytes": rows * (2 * case["H"] * Dh * es + plain + Hkv * _row_bytes(case) + back + 4),
                "flops": rows * (case["H"] + Hkv) * (5 * Dh + 3 * case["rot"]) + rows * 3 * plain}
    if kind == "convert":
        slots = _slots(case)
        return {"bytes": slots * (Hkv * _row_bytes(case) + plain * (2 if case["write"] else 1)), "flops": slots * plain}
    if kind == "compact":
        moved = case["a"] + (B - 1) * (max(1, case["a"] // 2) + case["a"]) / 2
        return {"bytes": moved * (2 * Hkv * _row_bytes(case) + plain), "flops": moved * plain}
    rows, H = _rows(case), case["H"]
    own_slots = _slots(case) + rows
    shared = case["phi"] + max(0, case["groups"] - 1) * (case["plo"] + case["phi"]) / 2
    seen = (case["plo"] + case["phi"]) / 2 + _slots(case) / B + rows / B / 2
    return {"bytes": 2 * es * rows * H * Dh + 16 * rows + (own_slots + shared) * Hkv * _row_bytes(case),
            "flops": 4 * rows * H * seen * Dh}


# ------------------------------------------------------------------------------ in 64 bits
def _grid(kind):
    """The sizes that an eight-bit type has, in rising order."""
    if kind == "int8":
        return [float(i) for i in range(128)]
    low = [m / 8 * 2.0 ** -6 for m in range(8)]
    return low + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8) if (e, m) != (8, 7)]


def _nearest(t, kind):
    """t rounded to a value of the type; halfway between two, to the one of even index."""
    grid = torch.tensor(_grid(kind), dtype=torch.float64, device="cuda")
    a = t.abs().clamp(max=TOP[kind])
    hi = torch.searchsorted(grid, a.contiguous()).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    down, up = a - grid[lo], grid[hi] - a
    take = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return torch.sign(t) * grid[take]


def _stored(x, kind):
    """What rows of 64-bit values come to in the cache: a scale held in 32 bits, quotients rounded to 32 bits."""
    scale = (x.abs().max(-1, keepdim=True).values.to(torch.float32).to(torch.float64) / TOP[kind]).to(torch.float32).to(torch.float64)
    t = torch.nan_to_num(x / scale, nan=0.0).to(torch.float32).to(torch.float64)
    return _nearest(t, kind) * scale


def _exact_append(s):
    c, half = s.case, s.case["rot"] // 2
    freq = torch.tensor([math.exp(-i / half * math.log(THETA)) for i in range(half)], dtype=torch.float64, device="cuda")
    first, second = (slice(0, half), slice(half, c["rot"])) if c["layout"] == HALF else (slice(0, c["rot"], 2), slice(1, c["rot"], 2))
    out = s.out.double()
    store = c["type"] in TOP
    k_out, v_out = (s.kw.double(), s.vw.double()) if store else (s.kc.double(), s.vc.double())
    for b in range(c["B"]):
        m, L = int(s.rows[b]), int(s.L[b])
        turn = torch.polar(torch.ones_like(freq), s.pos[b, :m].double()[:, None] * freq)[:, None]

        def made(x, weight):
            x = x.double()
            if weight is not None:
                x = weight.double() * x * torch.rsqrt(x.pow(2).sum(-1, keepdim=True) / c["Dh"] + EPS)
            x = x.clone()
            z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
            x[..., first], x[..., second] = z.real, z.imag
            return x

        out[b, :m] = made(s.q[b, :m], s.q_norm)
        k, v = made(s.k[b, :m], s.k_norm), s.v[b, :m].double()
        at = slice(0, m) if store else slice(L, L + m)
        k_out[b, :, at] = (_stored(k, c["type"]) if store else k).transpose(0, 1)
        v_out[b, :, at] = (_stored(v, c["type"]) if store else v).transpose(0, 1)
    return {"q": out, "k": k_out, "v": v_out}


def _exact_convert(s):
    c = s.case
    k, v = s.kw.double(), s.vw.double()
    for b in range(c["B"]):
        L = int(s.L[b])
        for h in range(c["Hkv"]):
            if c["write"]:
                k[b, h, :L], v[b, h, :L] = (_stored(x[b, h, :L].double(), c["type"]) for x in (s.k0, s.v0))
            else:
                k[b, h, :L] = s.kc[b, h, :L].to(torch.float64) * s.ks[b, h, :L, None].double()
                v[b, h, :L] = s.vc[b, h, :L].to(torch.float64) * s.vs[b, h, :L, None].double()
    return {"k": k, "v": v}


def _exact_compact(s):
    c = s.case
    k, v = s.kw.double(), s.vw.double()
    for b in range(c["B"]):
        for m in range(int(s.n_acc[b])):
            j = int(s.L[b]) + int(s.path[b, m + 1])
            k[b, :, m] = s.kc[b, :, j].to(torch.float64) * s.ks[b, :, j, None].double()
            v[b, :, m] = s.vc[b, :, j].to(torch.float64) * s.vs[b, :, j, None].double()
    return {"k": k, "v": v}


def _exact_attn(s):
    c = s.case
    Hkv, Dh = c["Hkv"], c["Dh"]
    G = c["H"] // Hkv
    out = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda")

    def real(x, scale, i, h, count):
        y = x[i, h, :count].to(torch.float64)
        return y if scale is None else y * scale[i, h, :count, None].double()

    for h in range(Hkv):
        for b in range(c["B"]):
            m, L = int(s.rows[b]), int(s.L[b])
            k, v = real(s.kc, s.ks, b, h, L + m), real(s.vc, s.vs, b, h, L + m)
            seen = L
            if c["groups"]:
                j = b // (c["B"] // c["groups"])
                k = torch.cat([real(s.pk, s.pks, j, h, int(s.P[j])), k])
                v = torch.cat([real(s.pv, s.pvs, j, h, int(s.P[j])), v])
                seen += int(s.P[j])
            q = s.q[b, :m, h * G: (h + 1) * G].double().reshape(m * G, Dh)
            x = q @ k.t().contiguous() * Dh ** -0.5
            hidden = torch.from_numpy(~s.path[b][:m, :m]).cuda().repeat_interleave(G, 0)
            x[:, seen:] = x[:, seen:].masked_fill(hidden, -math.inf)
            p = torch.exp(x - torch.logsumexp(x, 1, keepdim=True))
            out[b, :m, h * G: (h + 1) * G] = (p @ v).view(m, G, Dh)
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    return {"append": _exact_append, "convert": _exact_convert, "compact": _exact_compact, "attn": _exact_attn}[case["kind"]](s)


if __name__ == "__main__":
    for c in listed() + [draw(random.Random(i)) for i in range(4)]:
        print(c, work(c))
