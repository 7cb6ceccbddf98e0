"""Tree attention over caches of any type, and behind shared prefixes, on the GPU against a plain
64-bit implementation.

Tolerances, per element, from the roundings on the way: a score is a sum of Dh products in fp32 and up
to three factors, off by at most ds = (Dh + 3) 2^-24 scale sum |q_d k_d|, so a probability by 2 ds + 2^-20
of itself (numerator and sum; the exponential's and the factors' ulps in the 2^-20); in bf16 it then
enters the second product, times its value's scale, rounded: 2^-8 of itself at most; that product and
the merges add up to 2^-24 per term; the output's own rounding is 2^-8 (bf16) or 2^-24 of it."""
import math
import re

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TOP = {"int8": 127.0, "e4m3": 448.0}
KINDS = ["bf16", "f32", "e4m3", "int8"]


@pytest.fixture(scope="module")
def rt():
    from paper_2512_21857_amd import runtime
    assert torch.cuda.is_available()
    return runtime


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def bits(t):
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def tree_paths(n, rng):
    """[n][n] truth values: node j on the path from the root to node i of a random tree."""
    p = np.zeros((n, n), dtype=bool)
    for i in range(n):
        if i:
            p[i] = p[rng.integers(max(0, i - 12), i)]
        p[i, i] = True
    return p


def packed(paths, n):
    w = np.zeros((n, 2), dtype=np.uint64)
    for i, j in zip(*np.nonzero(paths)):
        w[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return w.view(np.int64)


def filled(g, kind, *shape):
    """Keys, values and scales of a cache, and what they stand for in 64 bits is codes times scales."""
    if kind not in TOP:
        return [torch.empty(*shape, device="cuda").normal_(generator=g).to(DT[kind]) for _ in range(2)] + [None, None]
    kv, scales = [], []
    for _ in range(2):
        x = torch.empty(*shape, device="cuda").normal_(generator=g)
        s = x.abs().amax(-1) / TOP[kind]
        t = (x / s[..., None]).clamp(-TOP[kind], TOP[kind])
        kv.append((t.round() if kind == "int8" else t).to(DT[kind]))
        scales.append(s)
    return kv + scales


def values(x, scale, *at):
    y = x[at].double()
    return y if scale is None else y * scale[at].double()[..., None]


class Case:
    """Inputs of one call; caches may be one layer of a larger allocation."""

    def __init__(self, rt, kind, H, Hkv, Dh, n, L, rows=None, tails=None, P=None, cap=None, pcap=None, layers=0, seed=1, q_scale=1.0):
        g, rng = gen(seed), np.random.default_rng(seed)
        self.kind, self.H, self.Hkv, self.Dh, self.n, self.L, self.P = kind, H, Hkv, Dh, n, L, P
        self.dtype = "f32" if kind == "f32" else "bf16"
        self.B = len(L)
        self.rows = rows or [max(1, n - b * (n // 3)) for b in range(self.B)]
        self.tails = tails or [min(n, r + (1 if b % 2 else 0)) for b, r in enumerate(self.rows)]
        self.cap = cap or max(l + t for l, t in zip(L, self.tails)) + 5
        at = (lambda t: None if t is None else t[:, 1]) if layers else (lambda t: t)
        shape = (self.B, layers, Hkv, self.cap, Dh) if layers else (self.B, Hkv, self.cap, Dh)
        self.t = [at(x) for x in filled(g, kind, *shape)]
        for b in range(self.B):
            # what lies behind the tail is never read
            for x in (self.t[:2] if kind not in TOP else self.t[2:]):
                x[b, :, L[b] + self.tails[b]:] = math.nan
        self.cache = rt.KVCache(*self.t)
        self.prefix = None
        if P is not None:
            shape = (len(P), layers, Hkv, pcap or max(P) + 3, Dh) if layers else (len(P), Hkv, pcap or max(P) + 3, Dh)
            self.pt = [at(x) for x in filled(g, kind, *shape)]
            for j in range(len(P)):
                for x in (self.pt[:2] if kind not in TOP else self.pt[2:]):
                    x[j, :, P[j]:] = math.nan
            self.prefix = rt.KVCache(*self.pt)
        self.q = (q_scale * torch.empty(self.B, n, H, Dh, device="cuda").normal_(generator=g)).to(DT[self.dtype])
        self.mask = torch.from_numpy(np.stack([packed(tree_paths(n, rng), n) for _ in range(self.B)])).cuda()
        self.scale = 1 / math.sqrt(Dh)

    def call(self, rt, **kw):
        kw = {**dict(prefix=self.prefix, prefix_len=None if self.P is None else i32(self.P)), **kw}
        return rt.cache_tree_attn(self.q, self.cache, i32(self.L), i32(self.rows), i32(self.tails), self.mask, **kw)

    def tail_see(self, b):
        m = self.mask[b].cpu().numpy().view(np.uint64)
        t = [[bool(int(m[i, j // 64]) >> (j % 64) & 1) for j in range(self.tails[b])] for i in range(self.rows[b])]
        return torch.tensor(t, dtype=torch.bool, device="cuda").view(self.rows[b], self.tails[b])

    def reference(self, b, h):
        """Outputs [rows][G][Dh] and their tolerances, in 64 bits."""
        m, G = self.rows[b], self.H // self.Hkv
        L = min(self.L[b], self.cap)
        T = min(self.L[b] + self.tails[b], self.cap)
        k, v = (values(x, s, b, h, slice(0, T)) for x, s in ((self.t[0], self.t[2]), (self.t[1], self.t[3])))
        see = torch.cat([torch.ones(m, L, dtype=torch.bool, device="cuda"), self.tail_see(b)[:, : T - L]], 1)
        if self.P is not None:
            j = b // (self.B // len(self.P))
            pk, pv = (values(x, s, j, h, slice(0, self.P[j])) for x, s in ((self.pt[0], self.pt[2]), (self.pt[1], self.pt[3])))
            k, v = torch.cat([pk, k]), torch.cat([pv, v])
            see = torch.cat([torch.ones(m, self.P[j], dtype=torch.bool, device="cuda"), see], 1)
        see = see.repeat_interleave(G, 0)
        q = self.q[b, :m, h * G: (h + 1) * G].double().reshape(m * G, self.Dh)
        x = (q @ k.t().contiguous() * self.scale).masked_fill(~see, -math.inf)
        k0, v0 = torch.nan_to_num(k, 0, 0, 0), torch.nan_to_num(v, 0, 0, 0)
        ds = torch.where(see, q.abs() @ k0.abs().t().contiguous(), torch.zeros_like(x))
        ds = (ds.amax(1, keepdim=True) if ds.shape[1] else torch.zeros(m * G, 1, device="cuda").double()) * (self.scale * (self.Dh + 3) * 2.0 ** -24)
        top = x.amax(1, keepdim=True) if x.shape[1] else torch.full((m * G, 1), -math.inf, device="cuda").double()
        e = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
        total = e.sum(1, keepdim=True)
        p = torch.where(~see | (total == 0), torch.zeros_like(e), e / total)     # an unseen slot has no weight
        # a value that is not finite counts only where it is seen
        pv = p @ v0
        for j in (~torch.isfinite(v)).any(1).nonzero().flatten().tolist():
            odd = ~torch.isfinite(v[j])
            pv = torch.where(see[:, j: j + 1] & odd[None], pv + p[:, j: j + 1] * v[j][None], pv)
        rel = 2 * ds + 2.0 ** -20 + (x.shape[1] + 8) * 2.0 ** -24 + (2.0 ** -8 if self.dtype == "bf16" else 0.0)
        tol = rel * (torch.nan_to_num(p) @ v0.abs()) + STEP[self.dtype] * pv.abs() + 1e-30
        return pv.view(m, G, self.Dh), tol.view(m, G, self.Dh)

    def check(self, rt, out=None, rest=None, **kw):
        if out is None:
            out = torch.full_like(self.q, 7.0)
            assert self.call(rt, out=out, **kw) is out
        G = self.H // self.Hkv
        for b in range(self.B):
            for h in range(self.Hkv):
                want, tol = self.reference(b, h)
                got = out[b, : self.rows[b], h * G: (h + 1) * G].double()
                same = (got == want) | (torch.isnan(got) & torch.isnan(want))
                bad = ~(same | ((got - want).abs() <= tol))
                assert not bad.any(), f"b={b} h={h}: {int(bad.sum())} of {bad.numel()}, off by {(got - want).abs()[bad].max().item():.3e}"
            left = torch.full_like(out, 7.0) if rest is None else rest
            assert torch.equal(bits(out[b, self.rows[b]:]), bits(left[b, self.rows[b]:]))
        return out


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H,Hkv,Dh,n,L", [
    (4, 4, 64, 1, [1]),
    (4, 4, 64, 1, [0]),                    # the row's own slot alone
    (32, 8, 128, 1, [700]),
    (20, 20, 64, 17, [300, 31]),
    (8, 8, 128, 61, [64, 32, 513]),
    (16, 2, 128, 61, [100, 33]),           # 488 rows of one key-value head
    (4, 4, 64, 128, [129, 0]),             # a tail of both mask words
    (8, 1, 64, 33, [95]),
    (6, 2, 128, 8, [5000]),                # many splits
])
def test_attn(rt, kind, H, Hkv, Dh, n, L):
    print(f"attn {kind} H={H}/{Hkv} Dh={Dh} n={n} L={L}", flush=True)
    Case(rt, kind, H, Hkv, Dh, n, L).check(rt)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H,Hkv,Dh,n,L,P", [
    (4, 4, 64, 1, [3, 5], [40]),
    (32, 8, 128, 1, [1, 500, 33, 64], [700]),
    (20, 20, 64, 17, [30, 31, 90, 2], [120, 65]),
    (8, 8, 128, 61, [64, 32, 70], [513]),          # 183 rows: two blocks of them behind the prefix
    (16, 2, 64, 40, [10, 0, 7], [33]),
    (4, 2, 64, 128, [129, 0], [1, 300]),           # a group of one sequence each
    (6, 2, 128, 5, [200, 1300], [4000]),           # many splits of either part
])
def test_attn_prefix(rt, kind, H, Hkv, Dh, n, L, P):
    print(f"prefix {kind} H={H}/{Hkv} Dh={Dh} n={n} L={L} P={P}", flush=True)
    Case(rt, kind, H, Hkv, Dh, n, L, P=P).check(rt)


@pytest.mark.parametrize("kind", KINDS)
def test_many_sequences_behind_one_prefix(rt, kind):
    """More sequences than a wave has lanes, some without rows, rows of one block from many of them."""
    B = 150
    c = Case(rt, kind, 2, 1, 64, 3, [b % 7 for b in range(B)], rows=[(b * 5) % 4 for b in range(B)], P=[77])
    print(f"many {kind}", flush=True)
    c.check(rt)


@pytest.mark.parametrize("kind", KINDS)
def test_the_largest_group(rt, kind):
    """4096 sequences behind one prefix, one more is refused."""
    B, Dh, P = 4096, 64, 70
    g = gen(11)
    cache, prefix = (rt.KVCache(*filled(g, kind, n, 1, s, Dh)) for n, s in ((B, 4), (1, P)))
    dt = DT["f32" if kind == "f32" else "bf16"]
    q = torch.empty(B, 1, 2, Dh, device="cuda").normal_(generator=g).to(dt)
    kv_len = torch.arange(B, dtype=torch.int32, device="cuda") % 4
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    mask = torch.zeros(B, 1, 2, dtype=torch.int64, device="cuda")
    mask[:, :, 0] = 1
    print(f"largest group {kind}", flush=True)
    out = rt.cache_tree_attn(q, cache, kv_len, one, one, mask, prefix=prefix, prefix_len=i32([P]))
    kd, vd = (values(x, s, slice(None), 0) for x, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
    pk, pv = (values(x, s, 0, 0) for x, s in ((prefix.k, prefix.k_scale), (prefix.v, prefix.v_scale)))
    k = torch.cat([pk[None].expand(B, -1, -1), kd], 1)
    v = torch.cat([pv[None].expand(B, -1, -1), vd], 1)
    see = torch.cat([torch.ones(B, P, dtype=torch.bool, device="cuda"), torch.arange(4, device="cuda")[None] <= kv_len[:, None]], 1)
    qd, scale = q[:, 0].double(), 1 / math.sqrt(Dh)
    x = ((qd[:, :, None] * k[:, None]).sum(-1) * scale).masked_fill(~see[:, None], -math.inf)
    w = torch.softmax(x, -1)
    want = (w[..., None] * v[:, None]).sum(2)
    ds = ((qd.abs()[:, :, None] * k.abs()[:, None]).sum(-1).amax(-1, keepdim=True)) * (scale * (Dh + 3) * 2.0 ** -24)
    rel = 2 * ds + 2.0 ** -20 + (P + 12) * 2.0 ** -24 + (0.0 if kind == "f32" else 2.0 ** -8)
    tol = rel * (w[..., None] * v.abs()[:, None]).sum(2) + STEP["f32" if kind == "f32" else "bf16"] * want.abs() + 1e-30
    assert ((out[:, 0].double() - want).abs() <= tol).all()
    more = rt.KVCache.zeros(B + 1, 1, 4, Dh, DT[kind])
    n = torch.ones(B + 1, dtype=torch.int32, device="cuda")
    with pytest.raises(RuntimeError, match="sequences a group"):
        rt.cache_tree_attn(torch.zeros(B + 1, 1, 2, Dh, dtype=dt, device="cuda"), more, n, n, n,
                           torch.zeros(B + 1, 1, 2, dtype=torch.int64, device="cuda"), prefix=prefix, prefix_len=i32([P]))


@pytest.mark.parametrize("kind", KINDS)
def test_many_rows_of_few_parts(rt, kind):
    """More than 2^18 groups of four outputs, whose parts meet several rows to a thread; row counts that are no
    multiple of them, one and none."""
    B = 9
    c = Case(rt, kind, 32, 32, 128, 61, [3 + 17 * b for b in range(B)], rows=[61, 60, 1, 0, 33, 32, 31, 17, 61], P=[130])
    print(f"many rows {kind}", flush=True)
    c.check(rt)


@pytest.mark.parametrize("kind", KINDS)
def test_nothing_to_see(rt, kind):
    """Rows without any slot give zeros, with and without a prefix; empty prefixes, trees and sequences."""
    print(f"nothing {kind}", flush=True)
    c = Case(rt, kind, 4, 2, 64, 5, [0, 0, 9, 0], rows=[5, 2, 0, 3], tails=[5, 0, 0, 3])
    c.mask[0, 2] = 0
    c.mask[3] = 0
    out = c.check(rt)
    assert not out[0, 2].any() and not out[1, :2].any() and not out[3, :3].any()
    c = Case(rt, kind, 4, 2, 64, 5, [0, 0, 9, 0], rows=[5, 2, 0, 3], tails=[5, 0, 0, 3], P=[0, 50])
    c.mask[0, 2] = 0
    c.mask[3] = 0
    out = c.check(rt)
    assert not out[0, 2].any() and not out[1, :2].any() and out[3, :3].any()
    c = Case(rt, kind, 4, 2, 64, 5, [300, 200], P=[0], pcap=40)
    c.check(rt)
    c.check(rt, out=c.call(rt, out=torch.full_like(c.q, 7.0), prefix=None, prefix_len=None))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("P", [None, [70]])
def test_not_finite_in_masked_slots(rt, kind, P):
    """Keys, values and scales that are not finite in tail slots, and what they do to rows that see them only."""
    print(f"odd values {kind} {P}", flush=True)
    for seed in (1, 2):
        c = Case(rt, kind, 4, 2, 64, 40, [45, 64], rows=[40, 33], tails=[40, 40], P=P, seed=seed)
        for b, (slot, what) in enumerate([(3, math.nan), (38, math.inf)]):
            at = c.L[b] + slot
            if kind in TOP:
                c.t[2][b, 0, at] = what
                c.t[3][b, 1, at + 1] = math.nan
                if kind == "e4m3":
                    c.t[1].view(torch.uint8)[b, 0, at - 2, 5] = 0x7f           # NaN codes
                    c.t[0].view(torch.uint8)[b, 1, at - 3, 9] = 0xff
            else:
                c.t[0][b, 0, at, 7] = math.nan
                c.t[1][b, 1, at, 3] = what
                c.t[1][b, 1, at + 1, 60] = -math.inf
        c.check(rt)


@pytest.mark.parametrize("kind", KINDS)
def test_not_finite_in_seen_slots(rt, kind):
    """In slots that every row sees, and for the step that repeats the last slot, an infinite value stays one."""
    print(f"seen odd values {kind}", flush=True)
    c = Case(rt, kind, 4, 2, 64, 3, [37], P=[41])
    for t, last in ((c.t, 36), (c.pt, 40)):
        if kind in TOP:
            t[3][0, 0, last] = math.inf if kind == "int8" else math.nan
            t[1].view(torch.uint8)[0, 0, last] = 3
        else:
            t[1][0, 0, last, 9] = math.inf
    c.check(rt)
    c = Case(rt, kind, 4, 2, 64, 3, [37], P=[41])
    c.q[0, 1, 2, 5] = math.nan              # a row that is not finite, beside others
    c.check(rt)


@pytest.mark.parametrize("kind", KINDS)
def test_places(rt, kind):
    """Layers of a larger cache, bounds below the slots, lengths past the bound, outputs in place, sharp softmax."""
    print(f"places {kind}", flush=True)
    c = Case(rt, kind, 8, 4, 64, 9, [60, 7, 90, 33], P=[50, 20], layers=3)
    c.check(rt)
    c = Case(rt, kind, 8, 4, 128, 9, [60, 7], P=[50], cap=600, pcap=500)
    c.check(rt, kv_cap=70, prefix_cap=50)
    c.check(rt)
    was = c.q.clone()
    out = c.call(rt, out=c.q)
    c.q = was
    c.check(rt, out=out, rest=was)
    for P in (None, [300]):
        c = Case(rt, kind, 8, 4, 128, 9, [600, 7], P=P, q_scale=12.0)
        c.check(rt)
    # more slots than the bound: those past it are not seen
    c = Case(rt, kind, 8, 4, 64, 9, [60, 7], tails=[9, 9], cap=80, P=[50])
    short = Case(rt, kind, 8, 4, 64, 9, [60, 7], tails=[9, 9], cap=80, P=[50])
    short.P, short.tails = [40], [5, 9]
    full = rt.cache_tree_attn(c.q, c.cache, i32(c.L), i32(c.rows), i32(c.tails), c.mask, kv_cap=65, prefix=c.prefix,
                              prefix_len=i32([50]), prefix_cap=40)
    assert torch.equal(bits(full[0, : c.rows[0]]), bits(short.call(rt, kv_cap=65, prefix_cap=40)[0, : c.rows[0]]))


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_slots_past_32_bits(rt, kind):
    """A long prefix and a long cache of one allocation whose elements and heads lie past 2^31."""
    print(f"far slots {kind}", flush=True)
    cap, Hkv, Dh = 9_000_000, 2, 128                   # 2^31.1 codes in all, the second head past 2^30
    c = Case(rt, kind, 2, Hkv, Dh, 2, [40], P=[50])
    big = [torch.zeros(2, Hkv, cap, Dh, dtype=torch.int8, device="cuda").view(DT[kind]) for _ in range(2)]
    scales = [torch.zeros(2, Hkv, cap, device="cuda") for _ in range(2)]
    far = cap - 60
    small, psmall = c.t, c.pt
    # the same rows, the last slots of a very long cache whose other rows weigh nothing beside them
    for x, s, t, ts, p, ps in ((big[0], scales[0], small[0], small[2], psmall[0], psmall[2]),
                               (big[1], scales[1], small[1], small[3], psmall[1], psmall[3])):
        n = c.L[0] + c.tails[0]
        x.view(torch.int8)[1, :, far: far + n] = t.view(torch.int8)[0, :, :n]
        s[1, :, far: far + n] = ts[0, :, :n]
        x.view(torch.int8)[0, :, far: far + 50] = p.view(torch.int8)[0, :, :50]
        s[0, :, far: far + 50] = ps[0, :, :50]
    own, pre = (rt.KVCache(*(t[i: i + 1] for t in big + scales)) for i in (1, 0))
    q = 40.0 * c.q
    got = rt.cache_tree_attn(q, own, i32([far + c.L[0]]), i32(c.rows), i32(c.tails), c.mask, prefix=pre, prefix_len=i32([far + 50]))
    # in 64 bits: the far slots, and 2 far others of score and value 0
    for h in range(Hkv):
        n = c.L[0] + c.tails[0]
        k = torch.cat([values(p, s, 0, h, slice(0, m)) for p, s, m in ((psmall[0], psmall[2], 50), (small[0], small[2], n))])
        v = torch.cat([values(p, s, 0, h, slice(0, m)) for p, s, m in ((psmall[1], psmall[3], 50), (small[1], small[3], n))])
        see = torch.cat([torch.ones(2, 50 + c.L[0], dtype=torch.bool, device="cuda"), c.tail_see(0)], 1)
        x = (q[0, :, h].double() @ k.t().contiguous() * c.scale).masked_fill(~see, -math.inf)
        top = x.amax(1, keepdim=True).clamp(min=0)
        e = torch.exp(x - top)
        total = e.sum(1, keepdim=True) + 2 * far * torch.exp(-top)
        want = e @ v / total
        # scores up to 40 times a usual one: 2 ds of them, the sum of 2 far equal terms in fp32 (each a rounding)
        ds = (q[0, :, h].double().abs() @ k.abs().t().contiguous()).amax(1, keepdim=True) * (c.scale * (Dh + 3) * 2.0 ** -24)
        tol = (2 * ds + 2.0 ** -8 + 2.0 ** -16) * (e / total @ v.abs()) + 2.0 ** -8 * want.abs() + 1e-6
        assert torch.all((got[0, :, h].double() - want).abs() <= tol)


def planned_parts(rt, c, **kw):
    """How many partial results a row may have in a call: what it asks for when it gets too little workspace."""
    try:
        c.call(rt, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"), **kw)
    except rt.abi.AdtError as e:
        need = int(re.search(r"< (\d+) bytes", str(e)).group(1))
        return need // (c.B * c.H * c.n * (c.Dh + 2) * 4)
    return 1


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H,Hkv,Dh,n,L,P,least", [
    (2, 2, 128, 61, [3000], None, 4),             # two tiles of 32 rows, units dealt out to several workgroups
    (2, 2, 128, 61, [2975, 40], None, 4),         # ends within a unit's first half; a sequence of one split
    (2, 1, 64, 17, [2113], None, 3),              # two tiles that two rows short of one share
    (8, 1, 64, 40, [5000, 33], None, 4),          # four tiles, three blocks of rows
    (4, 1, 128, 128, [4031], None, 4),            # a tail of four steps at the end of a split
    (4, 2, 64, 20, [70, 9, 300], [4000], 4),      # 120 rows behind a prefix of several splits, own slots of one
    (2, 1, 128, 61, [700, 5000], [4033, 90], 6),  # several splits of either part
])
def test_many_rows_of_several_splits(rt, kind, H, Hkv, Dh, n, L, P, least):
    """The keys of more than 32 rows dealt out to several workgroups, with tail slots that are not finite."""
    print(f"splits {kind} H={H}/{Hkv} Dh={Dh} n={n} L={L} P={P}", flush=True)
    c = Case(rt, kind, H, Hkv, Dh, n, L, P=P, seed=5)
    assert planned_parts(rt, c) >= least
    c.check(rt)
    for b in range(len(L)):
        at = c.L[b] + c.tails[b] - 1
        if kind in TOP:
            c.t[3][b, 0, at] = math.nan
            c.t[2][b, 0, at - 1] = math.nan
        else:
            c.t[1][b, 0, at, 5] = math.inf
            c.t[0][b, 0, at - 1, 7] = math.nan
    c.check(rt)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Dh", [64, 128])
def test_many_rows_of_several_parts(rt, kind, Dh):
    """More than 2^18 groups of four outputs that meet several rows to a thread, two parts a round: four, three and one
    of them in the groups' rows."""
    if kind == "f32":
        # (whose workgroups take 32 rows: so many of 64 dims never split)
        B, n, P = 8 * 128 // Dh, 32, [2500, 1200]
        c = Case(rt, kind, 32, 32, Dh, n, [3 + 7 * b for b in range(B)], rows=[32 - b % 5 * 7 for b in range(B)], P=P)
    else:
        B, n, P = 9, 61, [2500, 1800, 0]
        c = Case(rt, kind, 32, 32, Dh, n, [3 + 17 * b for b in range(B)], rows=[61, 60, 1, 0, 33, 32, 31, 17, 61], P=P)
    print(f"many parts {kind} Dh={Dh}", flush=True)
    assert B * 32 * n * Dh // 4 >= 1 << 18 and planned_parts(rt, c) >= (4 if kind != "f32" else 3 if Dh == 128 else 2)
    c.check(rt)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Dh", [64, 128])
def test_few_rows_of_many_parts(rt, kind, Dh):
    """More than eight parts of few rows, which groups of threads deal out, at either size of a head."""
    c = Case(rt, kind, 2, 1, Dh, 4, [6000, 3000], rows=[4, 3])
    print(f"few rows, many parts {kind} Dh={Dh}", flush=True)
    assert planned_parts(rt, c) > 8
    c.check(rt)


def few_bits(c, which, value):
    """Sets every value of a case's caches (which: 1, the values' tensors) to about `value`: of the dim's sign, a tenth of it less at most."""
    g = gen(31)
    for t in [c.t] + ([c.pt] if c.P is not None else []):
        x, sign = t[which], torch.where(torch.rand(c.Dh, device="cuda", generator=g) < 0.5, -1.0, 1.0)
        near = 1.0 - 0.1 * torch.rand(x.shape, device="cuda", generator=g)
        if c.kind in TOP:
            x.copy_((near * sign * TOP[c.kind]).to(DT[c.kind]))
            t[which + 2].masked_fill_(torch.isfinite(t[which + 2]), value / TOP[c.kind])
        else:
            x.copy_(torch.where(torch.isnan(x.float()), x.float(), near * sign * value))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H,Hkv,Dh,n,L,P", [
    (4, 2, 64, 5, [300, 9], None),            # up to 32 rows, one split
    (4, 2, 128, 4, [5000], None),             # several
    (8, 2, 64, 17, [90, 7], None),            # three tiles
    (2, 2, 128, 61, [3000], None),            # two tiles, several splits
    (8, 2, 64, 40, [70, 0, 300, 31], [700, 0]),
    (32, 32, 128, 61, [3, 20, 37, 54], [2500]),
])
def test_values_at_the_end_of_fp32(rt, kind, H, Hkv, Dh, n, L, P):
    """Values whose weighted sums leave fp32, though no mean of them does; and values as small."""
    print(f"large values {kind} H={H}/{Hkv} Dh={Dh} n={n} L={L} P={P}", flush=True)
    c = Case(rt, kind, H, Hkv, Dh, n, L, P=P, seed=6, q_scale=3.0)
    for value in (3e38, 2.0 ** 121, 1e-25):
        few_bits(c, 1, value)
        was = c.q.clone()
        c.check(rt)
        out = c.call(rt, out=c.q)
        c.q = was
        c.check(rt, out=out, rest=was)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("n,L,P", [(3, [300], None), (40, [70], None), (4, [5000], None), (40, [70, 33], [700])])
def test_small_values_beside_the_largest(rt, kind, n, L, P):
    """Dims of small values beside dims whose sums leave fp32."""
    print(f"small beside large {kind} n={n} L={L} P={P}", flush=True)
    c = Case(rt, kind, 4, 2, 64, n, L, P=P, seed=9)
    few_bits(c, 1, 3e38)
    for t in [c.t] + ([c.pt] if P else []):
        t[1][..., ::3] *= 2.0 ** -119
        t[1][..., ::3] *= 2.0 ** -119                       # (some 2^-110)
        assert t[1][..., ::3].any()
    out = c.check(rt)
    for b in range(c.B):
        for h in range(2):
            want, tol = c.reference(b, h)
            got = out[b, : c.rows[b], 2 * h: 2 * h + 2].double()
            # (without the allowance for what is far below 1)
            assert torch.all(((got - want).abs() <= tol - 1e-30 + 2.0 ** -149)[..., ::3])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_the_largest_values(rt, kind):
    """Every value the type's largest: so is every output."""
    print(f"largest values {kind}", flush=True)
    most = torch.finfo(DT[kind]).max
    for P, n in ((None, 3), ([900], 40)):
        c = Case(rt, kind, 4, 2, 64, n, [1000, 30], P=P, q_scale=3.0)
        for t in [c.t] + ([c.pt] if P else []):
            t[1].copy_(torch.where(torch.isnan(t[1]), t[1], torch.full_like(t[1], most)))
        c.check(rt)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,L,P", [(5, [300], None), (40, [70, 33], None), (61, [3000], None), (33, [20, 90], [800])])
def test_not_finite_among_the_largest_values(rt, kind, n, L, P):
    """A tail slot that is not finite, where the sums of the others' values leave fp32: rows that do not see it are the
    formula's, in those that do what it reaches is not finite; in place too."""
    print(f"odd among large {kind} n={n} L={L} P={P}", flush=True)
    c = Case(rt, kind, 4, 2, 64, n, L, P=P, seed=8, q_scale=2.0)
    few_bits(c, 1, 3e38)
    slots = [c.rows[b] // 2 for b in range(c.B)]
    for b, slot in enumerate(slots):
        if kind in TOP:
            c.t[3][b, :, L[b] + slot] = math.nan
        else:
            c.t[1][b, :, L[b] + slot, 7] = math.nan
    was = c.q.clone()
    for out in (torch.full_like(c.q, 7.0), c.q):
        c.call(rt, out=out)
        out, c.q = out.clone(), was
        for b, slot in enumerate(slots):
            see = c.tail_see(b)[:, slot]
            for h in range(2):
                want, tol = c.reference(b, h)
                got = out[b, : c.rows[b], 2 * h: 2 * h + 2].double()
                assert see.any() and not torch.isfinite(want[see]).all()
                assert torch.all(((got - want).abs() <= tol)[~see])
                odd = ~torch.isfinite(want)
                assert not torch.isfinite(got[odd]).any()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,L,P,at", [
    (2, [200], None, 3),              # one split, waves that meet
    (2, [6000], None, 3),             # several
    (40, [100], None, 3),             # two tiles
    (40, [6000], None, 70),
    (2, [50], [200], -3),             # in the prefix
    (70, [50], [3000], -3),
])
def test_not_finite_without_weight(rt, kind, n, L, P, at):
    """A seen slot whose value (scale) is not finite makes the row's output not finite, however little the slot weighs: the
    last slot before the tail, whose key is the queries', weighs 2^300 times as much."""
    print(f"weightless {kind} n={n} L={L} P={P}", flush=True)
    c = Case(rt, kind, 2, 2, 64, n, L, P=P, seed=7)
    c.q.copy_(c.q[:, :1].expand_as(c.q).clone())
    for h in range(2):
        key = c.q[0, 0, h].float() * 45
        if kind in TOP:
            s = key.abs().max() / TOP[kind]
            t = (key / s).clamp(-TOP[kind], TOP[kind])
            c.t[0][0, h, L[0] - 1] = (t.round() if kind == "int8" else t).to(DT[kind])
            c.t[2][0, h, L[0] - 1] = s
        else:
            c.t[0][0, h, L[0] - 1] = key.to(DT[kind])
    t, slot = (c.t, at) if at >= 0 else (c.pt, -at)
    if kind in TOP:
        t[3][0, 0, slot] = math.nan
    else:
        t[1][0, 0, slot, 9] = math.inf
        t[1][0, 0, slot, 33] = math.nan
    out = c.call(rt, out=torch.full_like(c.q, 7.0))
    for h in range(2):
        want, tol = c.reference(0, h)
        got = out[0, : c.rows[0], h: h + 1].double()
        odd = ~torch.isfinite(want)
        assert odd.any() == (h == 0) and torch.equal(~torch.isfinite(got), odd)
        assert torch.equal(torch.isnan(got)[torch.isnan(want)], torch.isnan(want)[torch.isnan(want)])
        assert torch.all(((got - want).abs() <= tol)[~odd])


@pytest.mark.parametrize("kind", KINDS)
def test_a_workspace_for_smaller_bounds(rt, kind):
    """A workspace for the largest bounds serves every smaller one, and a call without the prefix."""
    print(f"bounds {kind}", flush=True)
    for c in (Case(rt, kind, 32, 8, 128, 1, [40], cap=20000), Case(rt, kind, 8, 8, 64, 61, [40, 7, 0, 33], cap=2400, P=[60], pcap=2112),
              Case(rt, kind, 32, 8, 64, 1, [3, 40, 7, 0], cap=576, P=[60], pcap=20000)):
        ws = rt.cache_tree_attn_workspace(c.H, c.n, c.cache, prefix=c.prefix)
        pcaps = [None] if c.P is None else [c.prefix.slots, c.prefix.slots // 3, 700, 128, 60]
        for cap in (c.cap, c.cap * 5 // 8, c.cap // 5, 128, 101):
            for pcap in pcaps:
                c.check(rt, kv_cap=cap, prefix_cap=pcap, workspace=ws)
        if c.P is not None:
            P, c.P, c.prefix = c.P, None, None
            c.check(rt, workspace=ws)


@pytest.mark.parametrize("kind", KINDS)
def test_the_largest_group_of_large_heads(rt, kind):
    """4096 sequences behind one prefix, heads of 128: rows of one block from many of them, none in some."""
    B = 4096
    c = Case(rt, kind, 1, 1, 128, 2, [b % 3 for b in range(B)], rows=[b % 7 % 3 for b in range(B)], tails=[2] * B, P=[70])
    print(f"largest group, 128 {kind}", flush=True)
    out = torch.full_like(c.q, 7.0)
    c.call(rt, out=out)
    few, c.B = c.B, c.B
    for b in list(range(0, 40)) + list(range(2040, 2060)) + list(range(few - 20, few)):
        want, tol = c.reference(b, 0)
        assert torch.all((out[b, : c.rows[b]].double() - want).abs() <= tol)
        assert torch.all(out[b, c.rows[b]:] == 7.0)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_offsets_past_32_bits(rt, kind):
    """Slots of one head whose elements lie past 2^31, and sequences and groups whose elements lie past 2^32."""
    print(f"far offsets {kind}", flush=True)
    cap, Dh, B = 17_200_000, 128, 2                    # 2.2e9 codes a head, 4.4e9 in all
    c = Case(rt, kind, 2, 1, Dh, 2, [40, 33], rows=[2, 2], tails=[2, 2], P=[50, 41])
    far = cap - 60
    big = [[torch.zeros(B, 1, cap, Dh, dtype=torch.int8, device="cuda").view(DT[kind]) for _ in range(2)] +
           [torch.zeros(B, 1, cap, device="cuda") for _ in range(2)] for _ in range(2)]
    for x, t, n in ((big[0], c.t, [42, 35]), (big[1], c.pt, [50, 41])):
        for b in range(B):
            for i in range(4):
                y, z = (u.view(torch.int8) if u.element_size() == 1 else u for u in (x[i], t[i]))
                y[b, :, far: far + n[b]] = z[b, :, : n[b]]
    own, pre = (rt.KVCache(*x) for x in big)
    q = 40.0 * c.q
    for behind in (True, False):
        got = rt.cache_tree_attn(q, own, i32([far + l for l in c.L]), i32(c.rows), i32(c.tails), c.mask, prefix=pre if behind else None,
                                 prefix_len=i32([far + p for p in c.P]) if behind else None)
        # in 64 bits: the far slots, and the others of score and value 0
        for b in range(B):
            T = c.L[b] + 2
            k, v = (values(x, s, b, 0, slice(0, T)) for x, s in ((c.t[0], c.t[2]), (c.t[1], c.t[3])))
            see = torch.cat([torch.ones(2, c.L[b], dtype=torch.bool, device="cuda"), c.tail_see(b)], 1)
            if behind:
                pk, pv = (values(x, s, b, 0, slice(0, c.P[b])) for x, s in ((c.pt[0], c.pt[2]), (c.pt[1], c.pt[3])))
                k, v = torch.cat([pk, k]), torch.cat([pv, v])
                see = torch.cat([torch.ones(2, c.P[b], dtype=torch.bool, device="cuda"), see], 1)
            see = see.repeat_interleave(2, 0)
            rows = q[b].double().reshape(4, Dh)
            x = (rows @ k.t().contiguous() * c.scale).masked_fill(~see, -math.inf)
            top = x.amax(1, keepdim=True).clamp(min=0)
            e = torch.exp(x - top)
            total = e.sum(1, keepdim=True) + (2 if behind else 1) * far * torch.exp(-top)
            want = e @ v / total
            # scores up to 40 times a usual one: 2 ds of them; the weights of the others, one by one in fp32
            ds = (rows.abs() @ k.abs().t().contiguous()).amax(1, keepdim=True) * (c.scale * (Dh + 3) * 2.0 ** -24)
            tol = (2 * ds + 2.0 ** -8 + 2.0 ** -16) * (e / total @ v.abs()) + 2.0 ** -8 * want.abs() + 1e-6
            assert torch.all((got[b].double().reshape(4, Dh) - want).abs() <= tol)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_streams_and_graphs(rt, kind):
    """Another stream, two captured graphs that share a workspace, replayed between eager calls, each
    replay as the eager result."""
    print(f"graphs {kind}", flush=True)
    a = Case(rt, kind, 8, 4, 128, 9, [600, 7], P=[300], seed=1)
    b = Case(rt, kind, 8, 4, 128, 9, [20, 500], P=[300], seed=2)
    ws = rt.cache_tree_attn_workspace(8, 9, a.cache, prefix=a.prefix)
    ws2 = rt.cache_tree_attn_workspace(8, 9, b.cache, prefix=b.prefix)
    ws = ws if ws.numel() >= ws2.numel() else ws2
    args = [(c.q, c.cache, i32(c.L), i32(c.rows), i32(c.tails), c.mask) for c in (a, b)]
    pl = i32([300])
    eager = [rt.cache_tree_attn(*x, prefix=c.prefix, prefix_len=pl, out=torch.zeros_like(c.q), workspace=ws).clone()
             for x, c in zip(args, (a, b))]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        other = rt.cache_tree_attn(*args[0], prefix=a.prefix, prefix_len=pl, out=torch.zeros_like(a.q))
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(bits(other), bits(eager[0]))
    outs, graphs = [torch.zeros_like(c.q) for c in (a, b)], []
    for x, c, out in zip(args, (a, b), outs):
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            rt.cache_tree_attn(*x, prefix=c.prefix, prefix_len=pl, out=out, workspace=ws)
        graphs.append(g)
    for _ in range(4):
        for g, out, want in zip(graphs, outs, eager):
            out.zero_()
            g.replay()
            assert torch.equal(bits(out), bits(want))
        torch.cuda.synchronize()
    # lengths are read when the graph runs
    args[0][2].copy_(i32([3, 2]))
    outs[0].zero_()
    graphs[0].replay()
    assert torch.equal(bits(outs[0]), bits(rt.cache_tree_attn(*args[0], prefix=a.prefix, prefix_len=pl, out=torch.zeros_like(a.q))))


@pytest.mark.parametrize("kind", KINDS)
def test_same_as_the_attention_that_was_there(rt, kind):
    """Behind a prefix, what each sequence gives over one cache that holds prefix and own slots: bit for bit
    the same keys, so within the roundings of two orders of summation."""
    print(f"joined {kind}", flush=True)
    c = Case(rt, kind, 8, 4, 128, 9, [64, 7, 33], P=[200])
    joined = [None if t is None else torch.cat([torch.cat([p[:, :, :200]] * 3).view(torch.uint8) if p.element_size() == 1 else torch.cat([p[:, :, :200]] * 3),
                                                t.view(torch.uint8) if t.element_size() == 1 else t], 2) for t, p in zip(c.t, c.pt)]
    joined = [t if t is None or t.dtype != torch.uint8 else t.view(DT[kind]) for t in joined]
    both = rt.KVCache(*joined)
    out = rt.cache_tree_attn(c.q, both, i32([l + 200 for l in c.L]), i32(c.rows), i32(c.tails), c.mask, out=torch.full_like(c.q, 7.0))
    c.check(rt, out=out)
    if kind in ("bf16", "f32"):
        was = rt.tree_attn_weights(c.q, both.k, both.v, i32([l + 200 for l in c.L]), i32(c.rows), i32(c.tails), c.mask, both.slots,
                                   out=torch.full_like(c.q, 7.0))[0]
        c.check(rt, out=was)


@pytest.mark.parametrize("kind", ["e4m3", "int8", "bf16"])
def test_decoding_with_a_shared_prompt(rt, kind):
    """A run of them together: two images behind one prompt, whose rows are normalised, rotated and appended,
    attended to, an accepted path moved up, and the next tree; and the same with one cache of values read
    back, in 64 bits."""
    print(f"run {kind}", flush=True)
    B, H, Hkv, Dh, n, P = 2, 8, 4, 64, 12, 90
    g, rng = gen(11), np.random.default_rng(11)
    normal = lambda *s: torch.empty(*s, device="cuda").normal_(generator=g).bfloat16()  # noqa: E731
    prefix, cache = (rt.KVCache.zeros(m, Hkv, cap, Dh, DT[kind]) for m, cap in ((1, 128), (B, 200)))
    qn, kn = (1 + 0.2 * torch.empty(Dh, device="cuda").normal_(generator=g) for _ in range(2))
    freq, gain = rt.rope_freqs(Dh)
    prompt = [normal(1, P, h, Dh) for h in (H, Hkv, Hkv)]
    rt.norm_rope_append(*prompt, torch.arange(P, dtype=torch.int32, device="cuda")[None], i32([0]), i32([P]), freq, prefix, qn, kn)
    lens, plen = [0, 0], i32([P])
    kv_len = i32(lens)
    for step in range(4):
        rows = [n, n - 3 * (step % 3)]
        parent = np.full((B, n), -1, dtype=np.int32)
        for b in range(B):
            for i in range(1, rows[b]):
                parent[b, i] = max(parent[b, i - 1], int(rng.integers(max(0, i - 4), i)))
        mask, depth = rt.tree_masks(torch.from_numpy(parent).cuda(), i32(rows))
        pos = P + kv_len[:, None] + depth
        q, k, v = (normal(B, n, h, Dh) for h in (H, Hkv, Hkv))
        n_rows = i32(rows)
        qr = rt.norm_rope_append(q, k, v, pos.int(), kv_len, n_rows, freq, cache, qn, kn)
        out = rt.cache_tree_attn(qr, cache, kv_len, n_rows, n_rows, mask, prefix=prefix, prefix_len=plen)
        # the same from what the caches stand for
        c = Case.__new__(Case)
        c.kind, c.H, c.Hkv, c.Dh, c.n, c.L, c.P, c.B, c.rows, c.tails, c.cap = kind, H, Hkv, Dh, n, lens, [P], B, rows, rows, 200
        c.dtype, c.q, c.mask, c.scale = "bf16", qr, mask, Dh ** -0.5
        c.t, c.pt = ([x.k, x.v, x.k_scale, x.v_scale] for x in (cache, prefix))
        for b in range(B):
            for h in range(Hkv):
                want, tol = c.reference(b, h)
                got = out[b, : rows[b], h * 2: h * 2 + 2].double()
                assert torch.all((got - want).abs() <= tol)
        # a path from the root is accepted
        path, acc = np.zeros((B, n), dtype=np.int32), [0] * B
        for b in range(B):
            chain = [rows[b] - 1]
            while parent[b, chain[0]] > 0:
                chain.insert(0, int(parent[b, chain[0]]))
            acc[b] = len(chain)
            path[b, 1: 1 + len(chain)] = chain
        before = [x.clone() for x in (cache.k.view(torch.uint8) if kind != "bf16" else cache.k, cache.v.view(torch.uint8) if kind != "bf16" else cache.v)]
        rt.cache_compact(cache, kv_len, torch.from_numpy(path).cuda(), i32(acc), n - 1)
        for b in range(B):
            src = [lens[b] + int(x) for x in path[b, 1: 1 + acc[b]]]
            for now, was in zip((cache.k, cache.v), before):
                assert torch.equal(bits(now[b])[:, lens[b] + 1: lens[b] + 1 + acc[b]], bits(was[b])[:, src])
        lens = [l + 1 + a for l, a in zip(lens, acc)]
        kv_len = i32(lens)
