"""Operators of a long or bounded cache on the GPU against plain 64-bit implementations.

Tolerances count roundings: a value stored in bf16 is off by at most half a step, 2^-8 of its
size (8 significand bits kept), one in fp32 by 2^-24; what comes before the last rounding is
bounded where each test states its tolerance."""
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


# ---------------------------------------------------------------------------- rotary append
def rope_reference(x, pos, freq, gain, layout):
    """x [B][n][heads][Dh], pos [B][n], in 64 bits."""
    x = x.double().clone()
    rot = 2 * freq.numel()
    t = (pos.double()[..., None] * freq)[:, :, None]
    c, s = gain * torch.cos(t), gain * torch.sin(t)
    ia, ib = (range(0, rot // 2), range(rot // 2, rot)) if layout == "half" else (range(0, rot, 2), range(1, rot, 2))
    a, b = x[..., list(ia)], x[..., list(ib)]
    x[..., list(ia)], x[..., list(ib)] = a * c - b * s, a * s + b * c
    return x


def rope_case(rt, dtype, layout, B, n, H, Hkv, Dh, rot, fused=True, pos_max=5000, rows=None, scaling="plain",
              in_place=False, seed=1):
    g = gen(seed)
    cap = 40 + n
    if fused:
        qkv = normal(g, dtype, B, n, (H + 2 * Hkv) * Dh)
        q, k, v = (t.unflatten(-1, (-1, Dh)) for t in qkv.split([H * Dh, Hkv * Dh, Hkv * Dh], -1))
    else:
        q, k, v = (normal(g, dtype, B, n, h, Dh) for h in (H, Hkv, Hkv))
    kc, vc = normal(g, dtype, B, Hkv, cap, Dh), normal(g, dtype, B, Hkv, cap, Dh)
    pos = torch.randint(-3, pos_max, (B, n), generator=g, device="cuda", dtype=torch.int32)
    L = [(7 * b) % 40 for b in range(B)]
    rows = rows or [n - (b % 2) * (n // 3) for b in range(B)]
    freq, gain = rt.rope_freqs(rot, 10000.0, scaling, 8.0, 1024)
    out = q if in_place else torch.full((B, n, H, Dh), 3.0, dtype=DT[dtype], device="cuda")
    q0, out0, kc0, vc0 = q.clone(), out.clone(), kc.clone(), vc.clone()
    got = rt.rope_append(q, k, v, pos, i32(L), i32(rows), freq, kc, vc, layout=layout, gain=gain, out=out)
    assert got is out
    wq, wk = rope_reference(q0, pos, freq, gain, layout), rope_reference(k, pos, freq, gain, layout)
    # sine and cosine to about 2^-22 each (a quarter turn's remainder rounded to 24 bits, two ulp of
    # the function, the gain), two products and a sum: under 2^-20 of the pair's length; then the store
    pair = 2.0 ** -20 * 2 * gain * max(q0.abs().max().item(), k.abs().max().item())

    def near(a, ref):
        assert torch.all((a.double() - ref).abs() <= STEP[dtype] * ref.abs() + pair)

    for b in range(B):
        m, l = rows[b], L[b]
        near(out[b, :m], wq[b, :m])
        near(kc[b, :, l: l + m].transpose(0, 1), wk[b, :m])
        assert torch.equal(bits(vc[b, :, l: l + m].transpose(0, 1)), bits(v[b, :m]))
        for now, was in ((out[b, m:], out0[b, m:]), (kc[b, :, :l], kc0[b, :, :l]), (kc[b, :, l + m:], kc0[b, :, l + m:]),
                         (vc[b, :, :l], vc0[b, :, :l]), (vc[b, :, l + m:], vc0[b, :, l + m:])):
            assert torch.equal(bits(now), bits(was))
    # dims past the rotated ones pass unchanged
    assert torch.equal(bits(out[0, : rows[0], :, rot:]), bits(q0[0, : rows[0], :, rot:]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("B,n,H,Hkv,Dh,rot", [
    (1, 1, 32, 32, 128, 128),
    (3, 61, 20, 20, 64, 64),
    (2, 5, 32, 8, 128, 64),       # grouped heads, half of each head
    (2, 17, 3, 1, 96, 22),        # pairs that no 16 bytes hold: one value at a time
    (1, 700, 4, 2, 64, 48),       # more rows than a tree
    (5, 2, 1, 1, 2, 2),           # the smallest head
    (1, 9, 2, 2, 256, 256),       # the largest
])
def test_rope_append(rt, dtype, layout, B, n, H, Hkv, Dh, rot):
    print(f"rope {dtype} {layout} B={B} n={n} H={H}/{Hkv} Dh={Dh} rot={rot}", flush=True)
    rope_case(rt, dtype, layout, B, n, H, Hkv, Dh, rot)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scaling", ["linear", "base", "ramp"])
def test_rope_append_far_positions_and_scalings(rt, dtype, scaling):
    """Positions up to two million, where a float angle would be off by a tenth of a radian."""
    rope_case(rt, dtype, "half", 2, 33, 4, 4, 64, 64, pos_max=2_000_000, scaling=scaling)


def test_rope_append_in_place_and_contiguous_parts(rt):
    for layout in ("half", "interleaved"):
        rope_case(rt, "bf16", layout, 2, 6, 4, 2, 64, 32, fused=False, in_place=True)
        rope_case(rt, "f32", layout, 2, 6, 4, 2, 64, 32, fused=False)


def test_rope_append_no_rows(rt):
    rope_case(rt, "bf16", "half", 3, 4, 4, 4, 64, 64, rows=[0, 4, 0])


def test_rope_append_stops_at_the_capacity(rt):
    """Rows whose slots would pass the cache are rotated and not stored; nothing behind it changes."""
    g = gen(3)
    B, n, H, Dh, cap = 2, 4, 2, 64, 10
    q, k, v = (normal(g, "bf16", B, n, H, Dh) for _ in range(3))
    kc = torch.zeros(B, H, cap, Dh, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    freq, gain = rt.rope_freqs(Dh)
    pos = i32([[1, 2, 3, 4]] * B)
    out = rt.rope_append(q, k, v, pos, i32([8, -3]), i32([4, 4]), freq, kc, vc)
    want = rope_reference(q, pos, freq, gain, "half")
    assert torch.all((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5)
    assert torch.equal(bits(vc[0, :, 8:]), bits(v[0, :2].transpose(0, 1)))
    assert not vc[0, :, :8].any() and not vc[1].any() and not kc[1].any()


def test_rope_append_more_rows_than_a_launch(rt):
    """A launch has fewer than 2^32 threads a dimension: 2^24 rows and more take turns."""
    g = gen(12)
    n = (1 << 24) + 1003
    q, k, v = (normal(g, "bf16", 1, n, 1, 2) for _ in range(3))
    kc, vc = (torch.zeros(1, 1, n + 9, 2, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pos = torch.randint(0, 5000, (1, n), generator=g, device="cuda", dtype=torch.int32)
    freq, gain = rt.rope_freqs(2)
    out = rt.rope_append(q, k, v, pos, i32([5]), i32([n - 2]), freq, kc, vc, out=torch.full_like(q, 3.0))
    for got, x in ((out[0, : n - 2], q), (kc[0, 0, 5: n + 3, None], k)):
        want = rope_reference(x, pos, freq, gain, "half")[0, : n - 2]
        # (the pair's bound of the cases above: 2^-20 times its length, below 2 max|x|)
        assert torch.all((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19 * x.abs().max())
    assert torch.equal(bits(vc[0, 0, 5: n + 3]), bits(v[0, : n - 2, 0])) and not vc[0, 0, n + 3:].any()
    assert torch.all(out[0, n - 2:] == 3.0) and not kc[0, 0, n + 3:].any() and not kc[0, 0, :5].any()


def test_rope_inverse_positions_undo(rt):
    """Rotating by -pos what was rotated by pos gives the rows back, to four roundings of fp32."""
    g = gen(4)
    q, k, v = (normal(g, "f32", 1, 50, 2, 64) for _ in range(3))
    kc, vc = torch.zeros(1, 2, 60, 64, device="cuda"), torch.zeros(1, 2, 60, 64, device="cuda")
    freq, _ = rt.rope_freqs(64)
    pos = torch.arange(50, dtype=torch.int32, device="cuda")[None] * 4001
    a = rt.rope_append(q, k, v, pos, i32([0]), i32([50]), freq, kc, vc)
    b = rt.rope_append(a, k, v, -pos, i32([0]), i32([50]), freq, kc, vc)
    assert (b - q).abs().max().item() <= 2.0 ** -20 * 8


# ---------------------------------------------------------------------------- block means
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Dh", [64, 128])
@pytest.mark.parametrize("block,L", [(32, [1, 0, 31, 32, 33]), (64, [640, 700, 5, 64, 129]), (128, [1000, 127, 128, 384, 1])])
def test_block_keys(rt, dtype, Dh, block, L):
    g = gen(5)
    B, H, S = len(L), 3, 1003
    kc = normal(g, dtype, B, H, S, Dh)
    for b in range(B):
        kc[b, :, L[b]:] = math.nan                      # nothing behind the prefix is read
    out = rt.block_keys(kc, i32(L), block, out=torch.full((B, H, -(-S // block), Dh), 7.0, device="cuda"))
    for b in range(B):
        n = -(-L[b] // block)
        for j in range(n):
            rows = kc[b, :, j * block: min(L[b], (j + 1) * block)].double()
            # a sum of up to 128 terms in fp32 in any order, and the division
            tol = 2.0 ** -24 * (rows.abs().sum(1) / rows.shape[1] * rows.shape[1] + 1)
            assert torch.all((out[b, :, j].double() - rows.mean(1)).abs() <= tol)
        assert torch.all(out[b, :, n:] == 7.0)


def test_block_keys_from_a_start(rt):
    """Only the blocks from the start's on are written, in a layer of a larger cache."""
    g = gen(6)
    big = normal(g, "bf16", 2, 3, 4, 512, 64)
    kc = big[:, 1]
    L, start = [500, 300], [130, 300]
    full = rt.block_keys(kc, i32(L), 64)
    out = rt.block_keys(kc, i32(L), 64, start=i32(start), out=torch.full_like(full, 7.0))
    for b in range(2):
        j0, n = start[b] // 64, -(-L[b] // 64)
        assert torch.all(out[b, :, :j0] == 7.0) and torch.all(out[b, :, n:] == 7.0)
        assert torch.equal(out[b, :, j0:n], full[b, :, j0:n])
    assert torch.all((full[0, :, 0].double() - kc[0, :, :64].double().mean(1)).abs() <= 2.0 ** -18)


# ---------------------------------------------------------------------------- eviction
def kept_reference(w, L, budget, first, last):
    if L <= budget:
        return list(range(L))
    mid = sorted(range(first, L - last), key=lambda s: (w[s] != w[s], -w[s] if w[s] == w[s] else 0.0, s))
    keep = set(range(first)) | set(range(L - last, L)) | set(mid[: budget - first - last])
    return sorted(keep)


def evict_case(rt, dtype, B, slices, S, Dh, L, budget, first, last, weights=None, place=True, seed=9):
    g = gen(seed)
    kc, vc = normal(g, dtype, B, slices, S, Dh), normal(g, dtype, B, slices, S, Dh)
    w = torch.rand(B, slices, S, generator=g, device="cuda") if weights is None else weights(B, slices, S, g)
    k0, v0, w0 = kc.clone(), vc.clone(), w.clone()
    n_out = min(S, budget) + 3
    outs = {} if place else dict(k_out=torch.zeros(B, slices, n_out, Dh, dtype=DT[dtype], device="cuda"),
                                 v_out=torch.zeros(B, slices, n_out, Dh, dtype=DT[dtype], device="cuda"),
                                 weights_out=torch.zeros(B, slices, n_out, device="cuda"))
    kept, n = rt.kv_evict(kc, vc, w, i32(L), budget, first, last, **outs)
    ko, vo, wo = (kc, vc, w) if place else (outs["k_out"], outs["v_out"], outs["weights_out"])
    if not place:
        for now, was in ((kc, k0), (vc, v0), (w, w0)):
            assert torch.equal(bits(now), bits(was))
    assert n.tolist() == [min(l, budget) for l in L]
    wn = w0.cpu().numpy()
    for b in range(B):
        m = min(L[b], budget)
        for s in range(slices):
            want = kept_reference(wn[b, s], L[b], budget, first, last)
            assert kept[b, s, :m].tolist() == want
            assert torch.all(kept[b, s, m:] == -1)
            for now, was in ((ko, k0), (vo, v0), (wo, w0)):
                assert torch.equal(bits(now[b, s, :m]), bits(was[b, s, want]))
                if place:
                    assert torch.equal(bits(now[b, s, m:]), bits(was[b, s, m:]))
                else:
                    assert not now[b, s, m:].any()


@pytest.mark.parametrize("place", [True, False])
@pytest.mark.parametrize("dtype,B,slices,S,Dh,L,budget,first,last", [
    ("bf16", 2, 3, 700, 64, [700, 333], 256, 4, 32),
    ("f32", 2, 2, 300, 128, [299, 300], 299, 0, 0),           # one slot of one sequence goes
    ("bf16", 3, 2, 100, 128, [0, 1, 100], 1, 0, 0),           # empty, short, and a budget of one
    ("bf16", 1, 2, 5000, 64, [4777], 2049, 2049, 0),          # only the first slots
    ("bf16", 1, 2, 5000, 64, [4777], 2049, 0, 2049),          # only the last
    ("f32", 1, 1, 70000, 64, [69999], 40000, 3, 100),         # many rounds of the selection
    ("bf16", 2, 5, 64, 8, [64, 50], 33, 1, 1),                # rows of 16 bytes
    ("f32", 1, 2, 64, 12, [61], 17, 0, 16),                   # rows of 48 bytes
    ("bf16", 1, 2, 64, 64, [60], 1000, 5, 5),                 # a budget past the capacity
])
def test_kv_evict(rt, place, dtype, B, slices, S, Dh, L, budget, first, last):
    print(f"evict {dtype} B={B} slices={slices} S={S} Dh={Dh} L={L} budget={budget} place={place}", flush=True)
    evict_case(rt, dtype, B, slices, S, Dh, L, budget, first, last, place=place)


@pytest.mark.parametrize("kind", ["ties", "all_equal", "zeros_signed", "nonfinite", "negative", "tiny"])
def test_kv_evict_weight_orders(rt, kind):
    """Ties go to the lower slot; -0 equals 0; infinities are the ends of the order, NaN below all."""
    def weights(B, slices, S, g):
        w = torch.rand(B, slices, S, generator=g, device="cuda")
        if kind == "ties":
            return torch.floor(w * 5)
        if kind == "all_equal":
            return torch.full_like(w, 0.25)
        if kind == "zeros_signed":
            return torch.where(w < 0.5, torch.full_like(w, -0.0), torch.where(w < 0.9, torch.zeros_like(w), w))
        if kind == "nonfinite":
            w = torch.where(w < 0.3, torch.full_like(w, math.nan), w)
            w = torch.where(w > 0.9, torch.full_like(w, math.inf), w)
            return torch.where((w > 0.3) & (w < 0.5), torch.full_like(w, -math.inf), w)
        if kind == "negative":
            return w - 0.5
        return 1.0 + torch.floor(w * 300) * 2.0 ** -23       # apart in the last bits only
    for budget in (100, 700, 1500):
        evict_case(rt, "bf16", 2, 3, 2000, 64, [2000, 1777], budget, 3, 20, weights=weights)


@pytest.mark.parametrize("place", [True, False])
def test_kv_evict_more_than_65535_pieces(rt, place):
    """A budget of more than 65535 pieces of 128 rows, a workgroup each."""
    print(f"evict 8.4 M slots place={place}", flush=True)
    g = gen(13)
    S, first, last = 65535 * 128 + 5000, 7, 11
    budget = S - 1500
    kc, vc = (torch.randint(-30000, 30000, (1, 1, S, 8), generator=g, device="cuda").to(torch.int16).view(torch.bfloat16)
              for _ in range(2))
    w = torch.rand(1, 1, S, generator=g, device="cuda")
    k0, v0, w0 = kc.clone(), vc.clone(), w.clone()
    outs = {} if place else dict(k_out=torch.zeros_like(kc), v_out=torch.zeros_like(kc), weights_out=torch.zeros_like(w))
    kept, n = rt.kv_evict(kc, vc, w, i32([S]), budget, first, last, **outs)
    ko, vo, wo = (kc, vc, w) if place else outs.values()
    assert n.tolist() == [budget]
    # (a stable sort keeps the lower slot first among equal weights)
    order = torch.sort(w0[0, 0, first: S - last], descending=True, stable=True).indices[: budget - first - last] + first
    keep = torch.zeros(S, dtype=torch.bool, device="cuda")
    keep[order] = True
    keep[:first] = True
    keep[S - last:] = True
    want = keep.nonzero().flatten()
    assert torch.equal(kept[0, 0].long(), want)
    for now, was in ((ko, k0), (vo, v0), (wo, w0)):
        assert torch.equal(bits(now[0, 0, :budget]), bits(was[0, 0, want]))
        assert torch.equal(bits(now[0, 0, budget:]), bits(was[0, 0, budget:]) if place else torch.zeros_like(bits(now[0, 0, budget:])))


def ordered_weights(kind, g, *shape):
    w = torch.rand(*shape, generator=g, device="cuda")
    if kind == "ties":
        return torch.floor(w * 5)
    if kind == "all_equal":
        return torch.full_like(w, 0.25)
    if kind == "zeros_signed":
        return torch.where(w < 0.5, torch.full_like(w, -0.0), torch.where(w < 0.9, torch.zeros_like(w), w))
    if kind == "nonfinite":
        x = torch.where(w < 0.6, torch.full_like(w, math.nan), w)
        x = torch.where(w > 0.95, torch.full_like(w, math.inf), x)
        return torch.where((w > 0.6) & (w < 0.7), torch.full_like(w, -math.inf), x)
    if kind == "nan":
        return torch.full_like(w, math.nan)
    if kind == "negative":
        return w - 0.5
    if kind == "last_bits":
        return 1.0 + torch.floor(w * 300) * 2.0 ** -23
    return torch.exp(60 * (w - 0.5))                        # many exponents


# capacities at both ends of every form of the selection, and lengths that fill its rounds or just do not
@pytest.mark.parametrize("S,L", [(4096, [4096, 4095]), (4097, [4097, 4000]), (9000, [8999, 100]), (16384, [16384, 16383]),
                                 (16385, [16385, 2000]), (40000, [39999, 17]), (65536, [65536, 65535]),
                                 (65537, [65537, 65536]), (70000, [69999, 33000])])
@pytest.mark.parametrize("kind", ["ties", "all_equal", "zeros_signed", "nonfinite", "nan", "negative", "last_bits", "exponents"])
def test_kv_evict_weight_orders_at_every_capacity(rt, S, L, kind):
    """The selection has a form for each range of capacities; every one meets ties, zeros, infinities and
    NaN, with budgets of one slot, of some, of nearly all (into the NaN where there are any)."""
    print(f"evict orders S={S} L={L} {kind}", flush=True)
    g = gen(S + len(kind))
    B, slices = 2, 2
    kc, vc = (torch.randint(-30000, 30000, (B, slices, S, 8), generator=g, device="cuda").to(torch.int16).view(torch.bfloat16)
              for _ in range(2))
    w = ordered_weights(kind, g, B, slices, S)
    wn = w.cpu().numpy()
    for budget, first, last in ((1, 0, 0), (S // 3, 5, 64), (S - 1, 0, 0), (S - S // 8, 0, 7), (S // 2, 1, 0)):
        ko, vo = (torch.zeros(B, slices, budget, 8, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        kept, n = rt.kv_evict(kc, vc, w, i32(L), budget, first, last, k_out=ko, v_out=vo,
                              weights_out=torch.zeros(B, slices, budget, device="cuda"))
        assert n.tolist() == [min(l, budget) for l in L]
        for b in range(B):
            m = min(L[b], budget)
            for s in range(slices):
                want = np.arange(m)
                if L[b] > budget:
                    mid = wn[b, s, first: L[b] - last]
                    # by NaN last, then the larger weight (-0 and 0 alike), then the lower slot
                    order = np.lexsort((np.arange(mid.size), np.where(np.isnan(mid), 0, -mid), np.isnan(mid)))
                    keep = np.concatenate([np.arange(first), np.arange(L[b] - last, L[b]), order[: budget - first - last] + first])
                    want = np.sort(keep)
                assert np.array_equal(kept[b, s, :m].cpu().numpy(), want), (budget, b, s)
                at = torch.from_numpy(want).cuda()
                assert torch.equal(bits(ko[b, s, :m]), bits(kc[b, s, at])) and torch.equal(bits(vo[b, s, :m]), bits(vc[b, s, at]))


def test_kv_evict_length_in_place_and_layers(rt):
    """new_len is kv_len itself; the slices are those of one layer of a larger cache."""
    g = gen(10)
    big = normal(g, "bf16", 2, 3, 4, 200, 64)
    vbig = normal(g, "bf16", 2, 3, 4, 200, 64)
    w = torch.rand(2, 3, 4, 200, generator=g, device="cuda")
    b0, v0, w0 = big.clone(), vbig.clone(), w.clone()
    n = i32([180, 20])
    kept, _ = rt.kv_evict(big[:, 1], vbig[:, 1], w[:, 1], n, 50, 2, 8, new_len=n)
    assert n.tolist() == [50, 20]
    for l in (0, 2):
        assert torch.equal(bits(big[:, l]), bits(b0[:, l])) and torch.equal(w[:, l], w0[:, l])
    for s in range(4):
        want = kept_reference(w0[0, 1, s].tolist(), 180, 50, 2, 8)
        assert kept[0, s].tolist() == want
        assert torch.equal(bits(big[0, 1, s, :50]), bits(b0[0, 1, s, want]))
        assert torch.equal(bits(vbig[0, 1, s, :50]), bits(v0[0, 1, s, want]))
        assert torch.equal(bits(big[1, 1, s]), bits(b0[1, 1, s]))


def test_weights_compact(rt):
    g = gen(11)
    w = torch.rand(2, 3, 300, generator=g, device="cuda")
    w0 = w.clone()
    path = i32([[0, 1, 4, 9, 77], [0, 2, 0, 0, 0]])
    rt.weights_compact(w, i32([200, 290]), path, i32([4, 1]), 4)
    want = w0.clone()
    want[0, :, 201:205] = w0[0][:, [201, 204, 209, 277]]
    want[1, :, 291] = w0[1, :, 292]
    assert torch.equal(w, want)
    rt.weights_compact(w, i32([299, 299]), i32([[0, 1], [0, 5]]), i32([1, 1]), 1)      # past the capacity: left alone
    assert torch.equal(w, want)


# ---------------------------------------------------------------------------- the debug build
def test_lengths_past_the_capacity_are_recorded(rt, monkeypatch):
    """Device data that the host cannot check: the debug build records it, both builds stay in bounds."""
    from paper_2512_21857_amd import abi
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    B, H, Dh, n, cap = 1, 2, 64, 3, 64
    k, v = (torch.ones(B, H, cap, Dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.ones(B, n, H, Dh, dtype=torch.bfloat16, device="cuda")
    mask = torch.full((B, n, 2), 7, dtype=torch.int64, device="cuda")
    rows, w = i32(n), torch.ones(B, H, cap, device="cuda")
    freq, _ = rt.rope_freqs(Dh)
    means = torch.zeros(B, H, 2, Dh, device="cuda")

    def calls(L):
        yield lambda: rt.rope_append(q, q, q, i32(0, 1, 2)[None], i32(L), rows, freq, k, v)
        yield lambda: rt.block_keys(k, i32(L + 3), 32, out=means)
        yield lambda: rt.sparse_tree_attn(q, k, v, means, i32(L), rows, rows, mask, cap, 32, 1, 0, 1)
        yield lambda: rt.tree_attn_weights(q, k, v, i32(L), rows, rows, mask, cap)
        yield lambda: rt.kv_evict(k, v, w, i32(L + 3), 32)
        yield lambda: rt.weights_compact(w, i32(L), i32(0, 2)[None], i32(1), 1)

    for L, debug, recorded in ((61, True, False), (62, True, True), (62, False, False)):
        monkeypatch.setattr(rt, "lib", abi.lib_debug if debug else abi.lib)
        lib = rt.lib()
        stream = torch.cuda.current_stream().cuda_stream
        for i, call in enumerate(calls(L)):
            call()
            assert lib.adt_device_check(stream) == (abi.E_DEVICE_INVARIANT if recorded else abi.OK), (L, debug, i)
