"""Attention over a long cache on the GPU (chosen blocks, rated slots) against plain 64-bit
implementations.

Tolerances, per element, from the roundings on the way: a score is a sum of Dh products in fp32,
off by at most ds = Dh 2^-24 scale sum |q_d k_d|, so a probability by 2 ds + 2^-20 of itself
(numerator and sum; the exponential's and the factors' ulps in the 2^-20); in bf16 it then enters
the second product rounded, 2^-8 of itself at most; that product and the merges add up to 2^-24 per
term; the output's own rounding is 2^-8 (bf16) or 2^-24 of it."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def rt():
    from paper_2512_21857_amd import runtime
    assert torch.cuda.is_available()
    return runtime


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, dtype, *shape):
    return torch.empty(*shape, device="cuda").normal_(generator=g).to(DT[dtype])


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


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


class Case:
    """Inputs of one call; caches may be one layer of a larger allocation."""

    def __init__(self, dtype, H, Hkv, Dh, n, L, rows=None, cap=None, seed=1, layers=0, q_scale=1.0):
        g, rng = gen(seed), np.random.default_rng(seed)
        self.dtype, self.H, self.Hkv, self.Dh, self.n, self.L, self.B = dtype, H, Hkv, Dh, n, L, len(L)
        self.rows = rows or [max(1, n - b * (n // 3)) for b in range(self.B)]
        self.tails = [min(n, r + (1 if b % 2 else 0)) for b, r in enumerate(self.rows)]
        self.cap = cap or max(l + t for l, t in zip(L, self.tails)) + 5
        shape = (self.B, layers, Hkv, self.cap, Dh) if layers else (self.B, Hkv, self.cap, Dh)
        self.kbig, self.vbig = normal(g, dtype, *shape), normal(g, dtype, *shape)
        self.k, self.v = (self.kbig[:, 1], self.vbig[:, 1]) if layers else (self.kbig, self.vbig)
        self.q = (q_scale * torch.empty(self.B, n, H, Dh, device="cuda").normal_(generator=g)).to(DT[dtype])
        self.paths = [tree_paths(n, rng) for _ in range(self.B)]
        for b in range(self.B):
            # what lies behind the tail is never read
            self.k[b, :, L[b] + self.tails[b]:] = math.nan
            self.v[b, :, L[b] + self.tails[b]:] = math.nan
        self.mask = torch.from_numpy(np.stack([packed(p, n) for p in self.paths])).cuda()
        self.scale = 1 / math.sqrt(Dh)

    def dev(self):
        return i32(self.L), i32(self.rows), i32(self.tails), self.mask

    def tail_see(self, b):
        """[rows][tails]: what the rows see of the tree's slots, as the mask's bits say."""
        m = self.mask[b].cpu().numpy().view(np.uint64)
        t = [[bool(int(m[i, j // 64]) >> (j % 64) & 1) for j in range(self.tails[b])] for i in range(self.rows[b])]
        return torch.tensor(t, dtype=torch.bool, device="cuda").view(self.rows[b], self.tails[b])


def attend(c, b, h, see):
    """Outputs [rows][G][Dh], weights [rows][G][slots] and their tolerances, in 64 bits."""
    m, L, T, G = c.rows[b], c.L[b], c.L[b] + c.tails[b], c.H // c.Hkv
    q = c.q[b, :m, h * G: (h + 1) * G].double().reshape(m * G, c.Dh)
    k, v = c.k[b, h, :T].double(), c.v[b, h, :T].double()
    s = see.repeat_interleave(G, 0)
    k0, v0 = torch.nan_to_num(k, 0, 0, 0), torch.nan_to_num(v, 0, 0, 0)
    x = (q @ k.t().contiguous() * c.scale).masked_fill(~s, -math.inf)
    ds = torch.where(s, q.abs() @ k0.abs().t().contiguous(), torch.zeros_like(x)).amax(1, keepdim=True)
    ds = ds * (c.scale * c.Dh * 2.0 ** -24)
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(1, keepdim=True)
    p = torch.where(~s | (total == 0), torch.zeros_like(e), e / total)     # an unseen slot has no weight
    # a value that is not finite counts only where it is seen
    pv = p @ v0
    odd = ~torch.isfinite(v)
    if odd.any():
        for j in odd.any(1).nonzero().flatten().tolist():
            pv = torch.where(s[:, j: j + 1] & odd[j][None], pv + p[:, j: j + 1] * v[j][None], pv)
    terms = T + 8
    rel = 2 * ds + 2.0 ** -20 + terms * 2.0 ** -24 + (2.0 ** -8 if c.dtype == "bf16" else 0.0)
    tol = rel * (torch.nan_to_num(p) @ v0.abs()) + STEP[c.dtype] * pv.abs() + 1e-30
    wtol = torch.nan_to_num(p) * (2 * ds + 2.0 ** -20 + terms * 2.0 ** -24)
    return pv.view(m, G, c.Dh), tol.view(m, G, c.Dh), p.view(m, G, T), wtol.view(m, G, T)


def close(got, want, tol, what):
    got = got.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~(same | ((got - want).abs() <= tol))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, off by {(got - want).abs()[bad].max().item():.3e}"


def choose(c, b, h, means, block, n_sel, first, last):
    """[rows][blocks] truth values: the blocks each row takes."""
    m, G, L = c.rows[b], c.H // c.Hkv, c.L[b]
    n = -(-L // block)
    q = c.q[b, :m, h * G: (h + 1) * G].double().sum(1)
    score = (q @ means[b, h, :n].double().t().contiguous()).cpu().numpy()
    out = np.zeros((m, n), dtype=bool)
    for i in range(m):
        if n <= n_sel:
            out[i] = True
            continue
        mid = sorted(range(first, n - last), key=lambda j: (score[i, j] != score[i, j], -score[i, j], j))
        out[i, :first] = True
        out[i, n - last:] = True
        out[i, mid[: n_sel - first - last]] = True
    return out


def check_sparse(rt, c, block, n_sel, first=1, last=1, means=None, kv_cap=None, out=None):
    kv_len, n_q, n_tail, mask = c.dev()
    means = rt.block_keys(c.k, kv_len, block) if means is None else means
    out = torch.full_like(c.q, 3.0)
    sel = torch.full((c.B, c.n, c.Hkv, n_sel), -7, dtype=torch.int32, device="cuda")
    got = rt.sparse_tree_attn(c.q, c.k, c.v, means, kv_len, n_q, n_tail, mask, kv_cap or c.cap, block, n_sel, first, last,
                              out=out, sel=sel)
    assert got is out
    G = c.H // c.Hkv
    for b in range(c.B):
        m = c.rows[b]
        n = -(-c.L[b] // block)
        assert torch.all(out[b, m:] == 3.0) and torch.all(sel[b, m:] == -7)
        for h in range(c.Hkv):
            took = choose(c, b, h, means, block, n_sel, first, last)
            for i in range(m):
                want = np.nonzero(took[i])[0].tolist()
                assert sel[b, i, h].tolist() == want + [-1] * (n_sel - len(want)), (b, i, h)
            blk = torch.from_numpy(took).cuda().repeat_interleave(block, 1)[:, : c.L[b]]
            want, tol, _, _ = attend(c, b, h, torch.cat([blk, c.tail_see(b)], 1))
            close(out[b, :m, h * G: (h + 1) * G], want, tol, f"sparse b={b} h={h} L={c.L[b]} rows={m}")
    return out


SPARSE = [
    # H, Hkv, Dh, n, L, block, n_sel, first, last
    (8, 8, 128, 1, [1000], 64, 5, 1, 1),
    (32, 8, 128, 1, [3001, 40, 0], 64, 7, 1, 2),
    (8, 2, 64, 5, [513, 512, 1, 31], 32, 3, 1, 1),          # 20 rows: two tiles
    (4, 4, 64, 17, [300, 777], 32, 4, 0, 1),
    (4, 1, 128, 13, [2000, 129], 128, 4, 2, 2),             # only the ends
    (6, 2, 128, 61, [1500, 1499], 32, 12, 1, 1),            # 183 rows: three groups of 64
    (5, 5, 64, 128, [2345], 64, 9, 0, 0),
    (16, 1, 64, 128, [700], 32, 6, 1, 1),                   # 2048 rows of one key-value head
    (2, 2, 64, 3, [5000], 32, 150, 3, 5),                   # nearly all
    (2, 2, 128, 2, [100], 32, 40, 0, 0),                    # fewer blocks than asked for
    (3, 3, 64, 7, [64, 65, 63], 64, 1, 0, 1),               # one block
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,Dh,n,L,block,n_sel,first,last", SPARSE)
def test_sparse_tree_attn(rt, dtype, H, Hkv, Dh, n, L, block, n_sel, first, last):
    print(f"sparse {dtype} H={H}/{Hkv} Dh={Dh} n={n} L={L} block={block} sel={n_sel}", flush=True)
    check_sparse(rt, Case(dtype, H, Hkv, Dh, n, L, seed=n + len(L)), block, n_sel, first, last)


def test_sparse_more_blocks_than_lds_keys(rt):
    """More than 4096 blocks: the selection reads its keys anew; and many splits."""
    check_sparse(rt, Case("bf16", 2, 1, 64, 2, [140000], seed=4), 32, 33, 1, 1)


@pytest.mark.parametrize("kind", ["normal", "equal", "ties", "nan"])
def test_sparse_selection_in_rounds(rt, kind):
    """More than four rows over more than 1024 blocks: a workgroup selects for a row and reads its scores
    anew, here in three rounds of 2048, with ties and NaN across their ends."""
    print(f"sparse rounds {kind}", flush=True)
    c = Case("bf16", 2, 1, 64, 6, [140000], seed=4)
    means = torch.empty(1, 1, -(-c.cap // 32), 64, device="cuda").normal_(generator=gen(61))
    if kind == "equal":
        means[:] = means[:, :, :1]
    elif kind == "ties":
        means[:] = means[:, :, :7].repeat(1, 1, means.shape[2] // 7 + 1, 1)[:, :, : means.shape[2]]
    elif kind == "nan":
        means[:, :, 9:4370] = math.nan
        means[:, :, 2040:2056] = 1.0
    for n_sel, first, last in ((33, 1, 1), (1, 0, 0), (2500, 0, 2)):
        check_sparse(rt, c, 32, n_sel, first, last, means=means)


def test_sparse_layer_of_a_larger_cache(rt):
    check_sparse(rt, Case("bf16", 4, 2, 64, 9, [400, 333], layers=3), 32, 4)


def test_sparse_ties_take_the_lower_block(rt):
    c = Case("bf16", 4, 2, 64, 3, [640], seed=5)
    means = torch.zeros(1, 2, -(-c.cap // 32), 64, device="cuda")     # every score the same
    check_sparse(rt, c, 32, 6, 1, 1, means=means)
    means[:, :, 7] = math.nan                                          # NaN is below every number
    means[:, :, 3:5] = 1e30
    check_sparse(rt, c, 32, 6, 1, 1, means=means)
    means[:] = math.nan
    check_sparse(rt, c, 32, 6, 0, 0, means=means)


def test_sparse_near_scores_take_the_better_block(rt):
    """Means of two blocks apart by one fp32 step in one dim: double tells them apart for every row."""
    c = Case("f32", 2, 2, 64, 40, [640], seed=6)
    means = torch.empty(1, 2, -(-c.cap // 32), 64, device="cuda").normal_(generator=gen(60))
    means[:, :, 2:18] = means[:, :, 2:3]
    for j in range(2, 18):
        means[:, :, j, 0] = torch.tensor(1.0 + (j * 7 % 16) * 2.0 ** -23, device="cuda")
    check_sparse(rt, c, 32, 8, 1, 1, means=means)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sparse_values_that_are_not_finite(rt, dtype):
    """Infinities and NaN in keys and values reach only the rows that see their slots."""
    c = Case(dtype, 4, 2, 64, 20, [640, 0], rows=[20, 20], seed=7)
    means = rt.block_keys(c.k, i32(c.L), 32)
    c.v[0, :, 100] = math.nan
    c.v[0, :, 333, 5] = math.inf
    c.v[0, 1, 500, 9] = -math.inf
    c.v[0, :, 640 + 7] = math.inf               # a tree node's
    c.k[0, 0, 200] = math.nan
    c.v[1, :, 3] = math.nan
    c.k[1, 1, 9] = math.inf
    out = check_sparse(rt, c, 32, 5, 0, 1, means=means)
    assert torch.isfinite(out[0].float()).any() and not torch.isfinite(out[0].float()).all()


def test_sparse_rows_that_see_nothing(rt):
    c = Case("bf16", 4, 2, 128, 6, [0, 40], rows=[6, 6], seed=8)
    c.mask[0, 2:4] = 0
    c.mask[1, 0] = 0
    out = check_sparse(rt, c, 32, 1, 0, 1)
    assert not out[0, 2:4].any()


def test_sparse_no_rows_and_clamped_counts(rt):
    c = Case("bf16", 4, 2, 64, 6, [100, 90, 80], rows=[0, 6, 3], seed=9)
    check_sparse(rt, c, 32, 2)


# ---------------------------------------------------------------------------- rated slots
def check_weights(rt, c, decay=1.0, rated=False, w_in="given", place=False, seed=3):
    kv_len, n_q, n_tail, mask = c.dev()
    g = gen(seed)
    w = torch.rand(c.B, c.Hkv, c.cap, generator=g, device="cuda")
    for b in range(c.B):
        w[b, :, c.L[b]:] = math.nan                         # earlier weight of new slots is not read
    rating = torch.rand(c.B, c.n, generator=g, device="cuda") if rated else None
    w0 = w.clone()
    wo = w if place else torch.full_like(w, -5.0)
    out = torch.full_like(c.q, 3.0)
    got, gw = rt.tree_attn_weights(c.q, c.k, c.v, kv_len, n_q, n_tail, mask, c.cap, weights=None if w_in is None else w,
                                   decay=decay, row_weight=rating, out=out, weights_out=wo)
    assert got is out and gw is wo
    G = c.H // c.Hkv
    for b in range(c.B):
        m, L, T = c.rows[b], c.L[b], c.L[b] + c.tails[b]
        assert torch.all(out[b, m:] == 3.0)
        assert torch.all((wo[b, :, T:] == -5.0) | torch.isnan(wo[b, :, T:]))
        see = torch.cat([torch.ones(m, L, dtype=torch.bool, device="cuda"), c.tail_see(b)], 1)
        r = rating[b, :m].double() if rated else torch.ones(m, dtype=torch.float64, device="cuda")
        for h in range(c.Hkv):
            want, tol, p, ptol = attend(c, b, h, see)
            close(out[b, :m, h * G: (h + 1) * G], want, tol, f"rated b={b} h={h} L={L} rows={m}")
            add = (r[:, None, None] * p).sum((0, 1))
            atol = (r[:, None, None] * ptol).sum((0, 1)) + (m * G + 2) * 2.0 ** -24 * add
            if w_in is not None:
                add[:L] += decay * w0[b, h, :L].double()
                atol[:L] += 2.0 ** -23 * add[:L].abs()
            close(wo[b, h, :T], add, atol + 1e-30, f"weights b={b} h={h} L={L} rows={m}")
    return out, wo


RATED = [
    (8, 8, 128, 1, [1000]),
    (32, 8, 128, 1, [3001, 40, 0]),
    (8, 2, 64, 5, [513, 512, 1, 31]),
    (4, 4, 64, 17, [300, 777]),
    (4, 1, 128, 13, [2000, 129]),
    (6, 2, 128, 61, [1500, 1499]),
    (5, 5, 64, 128, [2345]),
    (16, 1, 64, 128, [700]),
    (40, 40, 64, 33, [256, 255, 257, 64, 0]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,Dh,n,L", RATED)
def test_tree_attn_weights(rt, dtype, H, Hkv, Dh, n, L):
    print(f"rated {dtype} H={H}/{Hkv} Dh={Dh} n={n} L={L}", flush=True)
    check_weights(rt, Case(dtype, H, Hkv, Dh, n, L, seed=n + len(L)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_attn_weights_forms(rt, dtype):
    c = Case(dtype, 8, 4, 64, 11, [200, 77], seed=12)
    check_weights(rt, c, decay=0.75, rated=True, place=True)
    check_weights(rt, c, w_in=None)
    check_weights(rt, c, decay=0.0, rated=True)
    check_weights(rt, Case(dtype, 4, 2, 64, 9, [400, 333], layers=3), decay=0.5)


def test_tree_attn_weights_peaked_and_low_scores(rt):
    """One slot takes nearly everything; and scores all far below zero (down to -1e4) still sum to one."""
    c = Case("bf16", 4, 2, 64, 7, [500], seed=13, q_scale=20.0)
    check_weights(rt, c)
    c = Case("f32", 2, 2, 64, 3, [90], seed=14)
    c.q[:] = -c.q.abs() * 1000
    c.k[:, :, :93] = c.k[:, :, :93].abs()
    out, w = check_weights(rt, c, w_in=None)
    assert abs(w[0, :, :93].double().sum().item() - 2 * 3) < 1e-4


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_attn_weights_values_that_are_not_finite(rt, dtype):
    c = Case(dtype, 4, 2, 64, 20, [150, 0], rows=[20, 20], seed=15)
    c.v[0, 0, 150 + 7] = math.inf
    c.v[0, 1, 150 + 3, 4] = math.nan
    c.k[0, 1, 150 + 9] = math.nan
    c.v[1, :, 5] = -math.inf
    c.k[1, 0, 2] = math.inf
    out, w = check_weights(rt, c)
    assert torch.isfinite(out[0].float()).any() and not torch.isfinite(out[0].float()).all()
    assert torch.isfinite(w[0, 0, :150]).all()


def test_tree_attn_weights_rows_that_see_nothing(rt):
    c = Case("bf16", 4, 2, 128, 6, [0, 40, 30], rows=[6, 6, 0], seed=16)
    c.mask[0, 2:4] = 0
    c.mask[1, 0] = 0
    out, w = check_weights(rt, c)
    assert not out[0, 2:4].any()


def test_attention_over_more_than_two_billion_elements(rt):
    """The last head of a cache whose elements pass 32 bits, by both attentions."""
    free = torch.cuda.mem_get_info()[0]
    if free < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    c = Case.__new__(Case)
    g = gen(17)
    c.dtype, c.H, c.Hkv, c.Dh, c.n, c.B, c.scale = "bf16", 18, 9, 128, 2, 1, 128 ** -0.5
    c.cap, c.L, c.rows, c.tails = 1_900_032, [1_900_000], [2], [2]
    c.k, c.v = (torch.empty(1, 9, c.cap, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert c.k.numel() > 2 ** 31
    for h in range(9):
        c.k[:, h].normal_(generator=g)
        c.v[:, h].normal_(generator=g)
    c.q = normal(g, "bf16", 1, 2, 18, 128)
    c.mask = torch.tensor([[[1, 0], [3, 0]]], dtype=torch.int64, device="cuda")
    kv_len, n_q, n_tail, mask = c.dev()
    out, w = rt.tree_attn_weights(c.q, c.k, c.v, kv_len, n_q, n_tail, mask, c.cap)
    see = torch.cat([torch.ones(2, c.L[0], dtype=torch.bool, device="cuda"), c.tail_see(0)], 1)
    want, tol, p, ptol = attend(c, 0, 8, see)
    close(out[0, :, 16:18], want, tol, "rated")
    add = p.sum((0, 1))
    close(w[0, 8, : add.numel()], add, ptol.sum((0, 1)) + 6 * 2.0 ** -24 * add, "weights")
    means = rt.block_keys(c.k, kv_len, 128)
    out = rt.sparse_tree_attn(c.q, c.k, c.v, means, kv_len, n_q, n_tail, mask, c.cap, 128, 20)
    took = choose(c, 0, 8, means, 128, 20, 1, 1)
    blk = torch.from_numpy(took).cuda().repeat_interleave(128, 1)[:, : c.L[0]]
    want, tol, _, _ = attend(c, 0, 8, torch.cat([blk, c.tail_see(0)], 1))
    close(out[0, :, 16:18], want, tol, "sparse")


def test_values_of_far_slots_and_heads(rt):
    """Values past 32 bits of elements, told apart by head and slot so that a wrong address shows: head h's
    are 2^h, four times that in the slots that take the attention, which lie at both ends, in the middle
    and around the element 2^31."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    g = gen(18)
    Hkv, Dh, L, block, n_sel = 9, 128, 1_900_000, 128, 20
    cap = L + 32
    k, v = (torch.empty(1, Hkv, cap, Dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert k.numel() > 2 ** 31
    q = normal(g, "bf16", 1, 1, Hkv, Dh)
    over = (2 ** 31 - (Hkv - 1) * cap * Dh) // Dh           # the last head's slot that holds the element 2^31
    peaks = [0, L // 2, over - 1, over, over + 1, L - 1]
    for h in range(Hkv):
        k[:, h].normal_(generator=g)
        v[:, h] = 2.0 ** h
        # a score of 200, where the others' standard deviation is |q| / sqrt(Dh), about one
        k[0, h, peaks] = (q[0, 0, h].float() * (200 * Dh ** 0.5 / q[0, 0, h].float().square().sum())).bfloat16()
        v[0, h, peaks] = 4 * 2.0 ** h
    mask = torch.ones(1, 1, 2, dtype=torch.int64, device="cuda")
    one = i32([1])
    means = rt.block_keys(k, i32([L]), block)
    # the peaks' weights are equal, the others' share is nothing (1.9e6 exp(10 - 200)): the output is 4 2^h to
    # the roundings of probabilities (2^-8) and output (2^-8); a mean score is 200 sqrt(Dh) / 128, above 17,
    # in a peak's block and about one elsewhere, so all their blocks are chosen
    want = 4 * 2.0 ** torch.arange(Hkv, device="cuda", dtype=torch.float64)
    out, w = rt.tree_attn_weights(q, k, v, i32([L]), one, one, mask, cap)
    assert torch.all((out[0, 0].double() - want[:, None]).abs() <= 2.0 ** -6 * want[:, None])
    assert torch.all((w[0, :, peaks].double().sum(1) - 1).abs() <= 2.0 ** -10)
    sel = torch.zeros(1, 1, Hkv, n_sel, dtype=torch.int32, device="cuda")
    near = rt.sparse_tree_attn(q, k, v, means, i32([L]), one, one, mask, cap, block, n_sel, sel=sel)
    assert torch.all((near[0, 0].double() - want[:, None]).abs() <= 2.0 ** -6 * want[:, None])
    for h in range(Hkv):
        assert {p // block for p in peaks} <= set(sel[0, 0, h].tolist())


# ---------------------------------------------------------------------------- much work at once
BATCHED = [
    # H, Hkv, Dh, n, L: 17..32, 33..64, 65..128 and more rows of a key-value head, for enough sequences to fill the CUs
    (32, 32, 128, 20, [1500, 64, 1339]),
    (32, 16, 64, 17, [3000, 100, 1500, 2049]),
    (64, 16, 64, 20, [3000, 2500, 1]),
    (64, 8, 64, 20, [3000, 2999, 0, 2048]),
    (16, 4, 128, 33, [4500, 4000, 4200, 128, 4499, 4300]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,Dh,n,L", BATCHED)
def test_tree_attn_weights_batched(rt, dtype, H, Hkv, Dh, n, L):
    print(f"rated {dtype} H={H}/{Hkv} Dh={Dh} n={n} L={L}", flush=True)
    check_weights(rt, Case(dtype, H, Hkv, Dh, n, L, seed=70 + n), decay=0.5)


@pytest.mark.parametrize("H,Hkv,Dh,n,L,block,n_sel", [
    (32, 32, 128, 20, [2500, 1300, 700], 64, 16),
    (32, 16, 64, 17, [4000, 100, 1500, 3900], 64, 30),
    (64, 16, 64, 20, [4000, 3000, 900], 128, 20),
    (64, 8, 64, 20, [5000, 4097, 0, 2048], 32, 70),
    (16, 4, 128, 5, [40000], 32, 40),                       # more than 1024 blocks, five rows
])
def test_sparse_tree_attn_batched(rt, H, Hkv, Dh, n, L, block, n_sel):
    print(f"sparse H={H}/{Hkv} Dh={Dh} n={n} L={L} block={block} sel={n_sel}", flush=True)
    check_sparse(rt, Case("bf16", H, Hkv, Dh, n, L, seed=80 + n), block, n_sel)


@pytest.mark.parametrize("Dh,n,L,block", [
    (64, 1, 524285, 32),                # the most blocks a call may have: 16384
    (64, 20, 524260, 32),
    (128, 4, 131060, 32),               # the most that four rows choose from in one launch: 4096
    (128, 1, 393100, 32),               # and one row: 12288
])
def test_sparse_at_the_limits_of_blocks(rt, Dh, n, L, block):
    print(f"sparse Dh={Dh} n={n} L={L}", flush=True)
    n_blk = -(-L // block)
    check_sparse(rt, Case("bf16", 2, 1, Dh, n, [L], cap=n_blk * block, seed=n + 40), block, 11)


@pytest.mark.parametrize("dtype,L", [("bf16", [300]), ("f32", [77]), ("bf16", [17000, 40])])
def test_tree_attn_weights_most_rows(rt, dtype, L):
    """8192 rows of one key-value head."""
    print(f"rated {dtype} 8192 rows L={L}", flush=True)
    check_weights(rt, Case(dtype, 64, 1, 64, 128, L, rows=[128] * len(L), seed=66), rated=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_short_prefixes_of_a_large_cache(rt, dtype):
    """The launch is sized for the capacity; hardly anything of it is used."""
    for n, H in ((1, 8), (3, 8), (20, 8), (70, 4)):
        c = Case(dtype, H, 4, 64, n, [33, 0, 129], cap=20000, seed=90 + n)
        check_weights(rt, c)
        check_sparse(rt, c, 32, 3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slots_past_the_capacity_are_not_seen(rt, dtype):
    """kv_cap below what the lengths say: the kernels stay within it (debug builds record it)."""
    for n, H in ((1, 8), (9, 4), (40, 8)):
        c = Case(dtype, H, 4, 64, n, [700, 300], rows=[n, n], seed=95 + n)
        cap = 690                                           # inside the first prefix, past all of the second
        k, v = c.k.clone(), c.v.clone()
        c.k[:, :, cap:] = math.nan
        c.v[:, :, cap:] = math.nan
        kv_len, n_q, n_tail, mask = c.dev()
        out = rt.sparse_tree_attn(c.q, c.k, c.v, rt.block_keys(k, kv_len, 32), kv_len, n_q, n_tail, mask, cap, 32, 22)
        rated, w = rt.tree_attn_weights(c.q, c.k, c.v, kv_len, n_q, n_tail, mask, cap,
                                        weights_out=torch.full((2, 4, c.cap), -5.0, device="cuda"))
        assert torch.all(w[0, :, cap:] == -5.0)
        assert torch.isfinite(out.float()).all()
        c.L, c.tails, c.k, c.v = [cap, 300], [0, n], k, v
        for b in range(2):
            for h in range(4):
                see = torch.cat([torch.ones(n, c.L[b], dtype=torch.bool, device="cuda"), c.tail_see(b)], 1)
                want, tol, p, ptol = attend(c, b, h, see)
                G = H // 4
                close(rated[b, :, h * G: (h + 1) * G], want, tol, f"rated b={b} h={h}")
                add = p.sum((0, 1))
                close(w[b, h, : add.numel()], add, ptol.sum((0, 1)) + (n * G + 2) * 2.0 ** -24 * add + 1e-30, "weights")
                # (22 blocks of 32 hold the second prefix, and the first up to the capacity)
                close(out[b, :, h * G: (h + 1) * G], want, tol, f"sparse b={b} h={h}")


# ---------------------------------------------------------------------------- how the calls are made
def _calls(rt, seed=21):
    """A call of every operator on inputs of its own: (function that runs it, its outputs)."""
    c = Case("bf16", 8, 4, 64, 9, [700, 333], seed=seed)
    kv_len, n_q, n_tail, mask = c.dev()
    g = gen(seed + 1)
    kc, vc = normal(g, "bf16", 2, 4, 900, 64), normal(g, "bf16", 2, 4, 900, 64)
    w = torch.rand(2, 4, c.cap, generator=g, device="cuda")
    means = torch.zeros(2, 4, -(-c.cap // 32), 64, device="cuda")
    freq, gain = rt.rope_freqs(64)
    pos = torch.randint(0, 9999, (2, 9), generator=g, device="cuda", dtype=torch.int32)
    kv, vv = normal(g, "bf16", 2, 9, 4, 64), normal(g, "bf16", 2, 9, 4, 64)
    o = dict(rot=torch.zeros_like(c.q), rated=torch.zeros_like(c.q), sparse=torch.zeros_like(c.q), kc=kc, vc=vc, means=means,
             sel=torch.zeros(2, 9, 4, 5, dtype=torch.int32, device="cuda"), w=torch.zeros_like(w),
             ko=torch.zeros(2, 4, 300, 64, dtype=torch.bfloat16, device="cuda"),
             vo=torch.zeros(2, 4, 300, 64, dtype=torch.bfloat16, device="cuda"), wo=torch.zeros(2, 4, 300, device="cuda"),
             kept=torch.zeros(2, 4, 300, dtype=torch.int32, device="cuda"), n=torch.zeros(2, dtype=torch.int32, device="cuda"))
    ws_s = rt.sparse_tree_attn_workspace(2, 8, 4, 64, 9, c.cap, 32, 5)
    ws_w = rt.tree_attn_weights_workspace(2, 8, 4, 64, 9, c.cap)

    def run():
        rt.rope_append(c.q, kv, vv, pos, kv_len, n_q, freq, kc, vc, gain=gain, out=o["rot"])
        rt.block_keys(c.k, kv_len, 32, out=means)
        rt.sparse_tree_attn(c.q, c.k, c.v, means, kv_len, n_q, n_tail, mask, c.cap, 32, 5, out=o["sparse"], sel=o["sel"],
                            workspace=ws_s)
        rt.tree_attn_weights(c.q, c.k, c.v, kv_len, n_q, n_tail, mask, c.cap, weights=w, out=o["rated"], weights_out=o["w"],
                             workspace=ws_w)
        rt.kv_evict(c.k, c.v, w, kv_len, 300, 2, 20, k_out=o["ko"], v_out=o["vo"], weights_out=o["wo"], kept=o["kept"],
                    new_len=o["n"])

    return run, o, c


def test_calls_are_captured_and_replayed(rt):
    """A graph of all operators, replayed with other inputs and eager work between the replays, gives
    what the eager calls give, bit for bit."""
    run, o, c = _calls(rt)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for r in range(4):
        c.q.copy_(normal(gen(100 + r), "bf16", *c.q.shape))
        run()
        torch.cuda.synchronize()
        want = {k: v.clone() for k, v in o.items()}
        for v in o.values():
            v.zero_()
        o["kc"].copy_(want["kc"])
        o["vc"].copy_(want["vc"])
        graph.replay()
        torch.cuda.synchronize()
        for k, v in o.items():
            assert torch.equal(v.nan_to_num(), want[k].nan_to_num()), (r, k)


def test_calls_on_another_stream_and_side_by_side(rt):
    """Two streams at work with workspaces of their own; the results are those of the default stream."""
    runs = [_calls(rt, seed) for seed in (31, 32)]
    wants = []
    for run, o, _ in runs:
        run()
        torch.cuda.synchronize()
        wants.append({k: v.clone() for k, v in o.items()})
    streams = [torch.cuda.Stream() for _ in runs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        for (run, _, _), s in zip(runs, streams):
            with torch.cuda.stream(s):
                run()
    torch.cuda.synchronize()
    for (_, o, _), want in zip(runs, wants):
        for k, v in o.items():
            assert torch.equal(v.nan_to_num(), want[k].nan_to_num()), k


def test_repeated_calls_give_the_same_bits(rt):
    """No sum depends on the order in which workgroups arrive."""
    for H, Hkv, n, L in ((32, 8, 1, [9000]), (16, 8, 16, [5000, 700]), (8, 8, 61, [2340])):
        c = Case("bf16", H, Hkv, 128, n, L, seed=40 + n)
        kv_len, n_q, n_tail, mask = c.dev()
        means = rt.block_keys(c.k, kv_len, 64)
        first = None
        for _ in range(5):
            out = rt.sparse_tree_attn(c.q, c.k, c.v, means, kv_len, n_q, n_tail, mask, c.cap, 64, 20, out=torch.zeros_like(c.q))
            o2, w = rt.tree_attn_weights(c.q, c.k, c.v, kv_len, n_q, n_tail, mask, c.cap, out=torch.zeros_like(c.q))
            got = [bits(out), bits(o2), bits(w)]
            first = first or got
            assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_dense_choice_equals_tree_attention(rt):
    """With all blocks taken, and one query head per key-value head, both attentions compute what
    tree_attn does: within the roundings of two bf16 results of the same sums."""
    c = Case("bf16", 6, 6, 128, 33, [500, 129], seed=50)
    c.k.nan_to_num_(0)
    c.v.nan_to_num_(0)
    kv_len, n_q, n_tail, mask = c.dev()
    want = rt.tree_attn(c.q, c.k, c.v, kv_len, n_q, n_tail, mask, c.cap, out=torch.zeros_like(c.q)).double()
    means = rt.block_keys(c.k, kv_len, 64)
    a = rt.sparse_tree_attn(c.q, c.k, c.v, means, kv_len, n_q, n_tail, mask, c.cap, 64, 100, out=torch.zeros_like(c.q))
    b, _ = rt.tree_attn_weights(c.q, c.k, c.v, kv_len, n_q, n_tail, mask, c.cap, out=torch.zeros_like(c.q))
    # each is within (2^-8 (rounded probabilities) + 2^-10) max|v| + 2^-8 |out| of the exact value
    vmax = c.v.abs().amax().item()
    for got in (a, b):
        assert torch.all((got.double() - want).abs() <= 2 * ((2.0 ** -8 + 2.0 ** -10) * vmax + 2.0 ** -8 * want.abs()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,n,L", [
    (8, 2, 1, [900, 0, 40]),            # few rows, splits merged by the last
    (4, 4, 20, [700, 64]),
    (8, 2, 61, [1500, 33]),             # 244 rows: several groups
    (4, 4, 61, [100]),                  # one split writes the output
])
def test_sparse_output_over_its_queries(rt, dtype, H, Hkv, n, L):
    print(f"sparse in place {dtype} H={H}/{Hkv} n={n} L={L}", flush=True)
    c = Case(dtype, H, Hkv, 64, n, L, seed=110 + n)
    kv_len, n_q, n_tail, mask = c.dev()
    means = rt.block_keys(c.k, kv_len, 32)
    want = rt.sparse_tree_attn(c.q, c.k, c.v, means, kv_len, n_q, n_tail, mask, c.cap, 32, 5, out=c.q.clone())
    out = c.q.clone()
    rt.sparse_tree_attn(out, c.k, c.v, means, kv_len, n_q, n_tail, mask, c.cap, 32, 5, out=out)
    assert torch.equal(bits(out), bits(want))


def test_refusals_of_the_wrappers(rt):
    """Tensors of other types, shapes, layouts or devices are refused before anything runs."""
    run, o, c = _calls(rt)
    kv_len, n_q, n_tail, mask = c.dev()
    means = rt.block_keys(c.k, kv_len, 32)
    good = dict(q=c.q, k=c.k, v=c.v, means=means, kv_len=kv_len, n_q=n_q, n_tail=n_tail, mask=mask)

    def sparse(**changed):
        a = {**good, **changed}
        return rt.sparse_tree_attn(*a.values(), c.cap, 32, 5)

    sparse()
    for bad in (dict(q=c.q.half()), dict(q=c.q.cpu()), dict(q=c.q.transpose(1, 2)), dict(k=c.k.float()), dict(v=c.v[..., ::2]),
                dict(v=c.v[:, :, :-1]), dict(means=means[:, :, :-1]), dict(means=means.double()), dict(kv_len=kv_len.long()),
                dict(kv_len=kv_len.cpu()), dict(n_q=n_q[:1]), dict(mask=mask[:, :-1]), dict(mask=mask.int())):
        with pytest.raises(ValueError):
            sparse(**bad)
    with pytest.raises(ValueError):
        rt.sparse_tree_attn(*good.values(), c.cap + 1, 32, 5)
    with pytest.raises(ValueError):
        rt.sparse_tree_attn(*good.values(), c.cap, 32, 5, sel=torch.zeros(2, 9, 4, 4, dtype=torch.int32, device="cuda"))
    from paper_2512_21857_amd import abi
    with pytest.raises(abi.AdtError):
        rt.sparse_tree_attn(*good.values(), c.cap, 32, 5, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    w = torch.rand(2, 4, c.cap, device="cuda")
    for bad in (dict(weights=w.double()), dict(weights=w[:, :, :-1]), dict(weights=w, weights_out=w[:, :, ::1].transpose(0, 1)),
                dict(row_weight=torch.ones(2, 8, device="cuda")), dict(out=c.q[:, :5])):
        with pytest.raises(ValueError):
            rt.tree_attn_weights(c.q, c.k, c.v, kv_len, n_q, n_tail, mask, c.cap, **bad)
    for bad in (dict(k_out=c.k), dict(kept=torch.zeros(2, 4, 9, dtype=torch.int32, device="cuda")),
                dict(k_out=o["ko"][:, :, :5], v_out=o["vo"][:, :, :5], weights_out=o["wo"])):
        with pytest.raises(ValueError):
            rt.kv_evict(c.k, c.v, w, kv_len, 300, **bad)


# ---------------------------------------------------------------------------- together
def test_bounded_cache_decoding(rt):
    """Decoding over a bounded cache, operator by operator against 64 bits: in every cycle a tree's rows are
    rotated at their own positions and appended, attend to all slots and rate them, attend to chosen
    blocks, an accepted path is compacted, with its weights, and the cache is cut to its budget, so that
    slots and positions part."""
    from paper_2512_21857_amd import abi
    B, H, Hkv, Dh, n, cap, budget, block = 2, 4, 2, 64, 7, 256, 96, 32
    g, rng = gen(60), np.random.default_rng(60)
    kc, vc = (torch.zeros(B, Hkv, cap, Dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w = torch.zeros(B, Hkv, cap, device="cuda")
    freq, gain = rt.rope_freqs(Dh, scaling="ramp", factor=4.0, orig_len=512)
    kv_len, seen = i32([0, 0]), [0, 0]
    c = Case.__new__(Case)
    c.dtype, c.H, c.Hkv, c.Dh, c.n, c.B, c.cap, c.scale = "bf16", H, Hkv, Dh, n, B, cap, Dh ** -0.5
    c.k, c.v = kc, vc
    cut = 0
    for cycle in range(40):
        parent = np.full((B, n), -1, dtype=np.int32)
        for b in range(B):
            for i in range(1, n):
                parent[b, i] = rng.integers(max(0, i - 3), i)
        c.rows = [n, n - cycle % 3]
        c.tails = c.rows
        c.L = kv_len.tolist()
        n_rows = i32(c.rows)
        c.mask, depth = rt.tree_masks(torch.from_numpy(parent).cuda(), n_rows)
        pos = i32(seen)[:, None] + depth
        qkv = normal(g, "bf16", B, n, (H + 2 * Hkv) * Dh)
        q, k, v = (t.unflatten(-1, (-1, Dh)) for t in qkv.split([H * Dh, Hkv * Dh, Hkv * Dh], -1))
        c.q = rt.rope_append(q, k, v, pos, kv_len, n_rows, freq, kc, vc, gain=gain)
        t = (pos.double()[..., None] * freq)[:, :, None]
        half = Dh // 2
        a, b2 = k.double()[..., :half], k.double()[..., half:]
        rot = gain * torch.cat([a * t.cos() - b2 * t.sin(), a * t.sin() + b2 * t.cos()], -1)
        for b in range(B):
            got = kc[b, :, c.L[b]: c.L[b] + c.rows[b]].transpose(0, 1).double()
            assert torch.all((got - rot[b, : c.rows[b]]).abs() <= 2.0 ** -8 * rot[b, : c.rows[b]].abs() + 1e-4)
        w0 = w.clone()
        out, _ = rt.tree_attn_weights(c.q, kc, vc, kv_len, n_rows, n_rows, c.mask, cap, weights=w, decay=0.9)
        means = rt.block_keys(kc, kv_len, block)
        near = rt.sparse_tree_attn(c.q, kc, vc, means, kv_len, n_rows, n_rows, c.mask, cap, block, 3)
        for b in range(B):
            m, L, G = c.rows[b], c.L[b], H // Hkv
            see = torch.cat([torch.ones(m, L, dtype=torch.bool, device="cuda"), c.tail_see(b)], 1)
            for h in range(Hkv):
                want, tol, p, ptol = attend(c, b, h, see)
                close(out[b, :m, h * G: (h + 1) * G], want, tol, f"cycle {cycle} rated")
                add = p.sum((0, 1))
                add[:L] += 0.9 * w0[b, h, :L].double()
                close(w[b, h, : L + m], add, ptol.sum((0, 1)) + 2.0 ** -19 * (add + 1), f"cycle {cycle} weights")
                if L:
                    took = choose(c, b, h, means, block, 3, 1, 1)
                    blk = torch.from_numpy(took).cuda().repeat_interleave(block, 1)[:, :L]
                    want, tol, _, _ = attend(c, b, h, torch.cat([blk, c.tail_see(b)], 1))
                    close(near[b, :m, h * G: (h + 1) * G], want, tol, f"cycle {cycle} sparse")
        # the path to a random node is accepted
        path, n_acc = np.zeros((B, n), dtype=np.int32), []
        for b in range(B):
            nodes, i = [], int(rng.integers(0, c.rows[b]))
            while i > 0:
                nodes.append(i)
                i = parent[b, i]
            path[b, 1: len(nodes) + 1] = nodes[::-1]
            n_acc.append(len(nodes))
        kb, wb = kc.clone(), w.clone()
        rt.kv_compact(kc, vc, kv_len, torch.from_numpy(path).cuda(), i32(n_acc), n - 1)
        rt.weights_compact(w, kv_len, torch.from_numpy(path).cuda(), i32(n_acc), n - 1)
        for b in range(B):
            src = [c.L[b] + path[b, m] for m in range(n_acc[b] + 1)]
            assert torch.equal(bits(kc[b, :, c.L[b]: c.L[b] + n_acc[b] + 1]), bits(kb[b, :, src]))
            assert torch.equal(w[b, :, c.L[b]: c.L[b] + n_acc[b] + 1], wb[b, :, src])
            seen[b] += n_acc[b] + 1
        kv_len = kv_len + 1 + i32(n_acc)
        before, kb, wb = kv_len.tolist(), kc.clone(), w.clone()
        kept, _ = rt.kv_evict(kc, vc, w, kv_len, budget, 4, 16, new_len=kv_len)
        for b in range(B):
            m = min(before[b], budget)
            assert kv_len.tolist()[b] == m
            cut += before[b] > budget
            for h in range(Hkv):
                keep = kept[b, h, :m].tolist()
                assert keep == sorted(keep) and len(set(keep)) == m
                if before[b] > budget:
                    assert keep[:4] == [0, 1, 2, 3] and keep[-16:] == list(range(before[b] - 16, before[b]))
                    lost = [s for s in range(before[b]) if s not in set(keep)]
                    assert max(wb[b, h, lost].tolist()) <= min(wb[b, h, keep[4:-16]].tolist())
                assert torch.equal(bits(kc[b, h, :m]), bits(kb[b, h, keep])) and torch.equal(w[b, h, :m], wb[b, h, keep])
    assert cut > 10 and min(seen) > budget      # the walk reached what it is for
    assert abi.lib().adt_device_check(None) == abi.OK
