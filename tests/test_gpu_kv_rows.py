"""Rows into, out of and within caches of any type on the GPU against plain 64-bit implementations.

Tolerances count roundings: a value stored in bf16 is off by at most half a step, 2^-8 of its size,
one in fp32 by 2^-24.  Queries are made in fp32: the sum of squares (up to 32 lanes' 8 terms, in a
tree), the factor's division and root, the gain, sine and cosine (rounded from double) and the two
products and the sum of a pair come to under 16 roundings, 2^-20 of the pair's length.  Keys are made in
double, where the two sides differ by 2^-48 or so, so codes and scales have to be the formula's: they
would differ only where a quotient lay that near a border between two codes, which none of the inputs'
does."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TOP = {"int8": 127.0, "e4m3": 448.0}


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
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def codes_of(x, kind):
    """(values of the codes, scales) that rows x (64 bits) come to in eight bits."""
    bad = ~torch.isfinite(x.float()).all(-1)
    x = torch.where(bad[..., None], torch.zeros_like(x), x)
    scale = (x.float().abs().amax(-1).double() / TOP[kind]).float()
    t = torch.where(scale[..., None] > 0, x / scale.double()[..., None], torch.zeros_like(x)).float().double()
    t = t.clamp(-TOP[kind], TOP[kind])
    if kind == "e4m3":
        step = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
        t = torch.round(t / step) * step
    else:
        t = torch.round(t)
    return t, torch.where(bad, torch.full_like(scale, math.nan), scale)


def new_cache(rt, g, kind, B, heads, cap, Dh, layers=0):
    """A cache of random contents; with layers, the second layer of a larger one."""
    shape = (B, layers, heads, cap, Dh) if layers else (B, heads, cap, Dh)
    at = (lambda t: t[:, 1]) if layers else (lambda t: t)
    if kind not in TOP:
        return rt.KVCache(*(at(normal(g, kind, *shape)) for _ in range(2)))
    kv = [torch.randint(-120, 120, shape, device="cuda", generator=g).to(torch.int8) for _ in range(2)]
    kv = [at(torch.where(t == -1, torch.zeros_like(t), t).view(DT[kind])) for t in kv]      # (no NaN of e4m3)
    return rt.KVCache(*kv, *(at(torch.rand(shape[:-1], device="cuda", generator=g)) for _ in range(2)))


def parts(c):
    return [t for t in (c.k, c.v, c.k_scale, c.v_scale) if t is not None]


def copies(c):
    return [t.clone() for t in parts(c)]


def rest_same(now, was, b, slots):
    """Every slot of sequence b but `slots` holds what it held."""
    keep = torch.ones(now[0].shape[2], dtype=torch.bool, device="cuda")
    keep[slots] = False
    for x, y in zip(now, was):
        assert torch.equal(bits(x[b])[:, keep], bits(y[b])[:, keep])


def made(x, w, eps, pos, freq, gain, layout):
    """x [B][n][heads][Dh] normalised (w not None) and rotated, in 64 bits."""
    x = x.double().clone()
    if w is not None:
        x = x * w.double() / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    length = x.clone()
    rot = 2 * freq.numel()
    t = (pos.double()[..., None] * freq)[:, :, None]
    c, s = gain * torch.cos(t), gain * torch.sin(t)
    ia, ib = (range(0, rot // 2), range(rot // 2, rot)) if layout == "half" else (range(0, rot, 2), range(1, rot, 2))
    ia, ib = list(ia), list(ib)
    a, b = x[..., ia], x[..., ib]
    x[..., ia], x[..., ib] = a * c - b * s, a * s + b * c
    length[..., ia] = length[..., ib] = gain * torch.hypot(a, b)
    return x, length.abs()


def append_case(rt, dtype, kind, norm, layout, B, n, H, Hkv, Dh, rot, fused=True, first=0, gain=1.0, eps=1e-5, cap=None, layers=0,
                rows=None, in_place=False, seed=1, edit=None):
    g = gen(seed)
    cap = cap or 40 + n
    eps = float(np.float32(eps))            # the call takes it in fp32 (1e-5 is not one: off by 2^-26 of it)
    if fused:
        qkv = 2 * normal(g, dtype, B, n, (H + 2 * Hkv) * Dh)
        q, k, v = (t.unflatten(-1, (-1, Dh)) for t in qkv.split([H * Dh, Hkv * Dh, Hkv * Dh], -1))
    else:
        q, k, v = (2 * normal(g, dtype, B, n, h, Dh) for h in (H, Hkv, Hkv))
    if edit:
        edit(k, v)
    wq = wk = None
    if norm != "none":
        wq, wk = (1 + 0.3 * normal(g, "f32", *([h] if norm == "heads" else []), Dh) for h in (H, Hkv))
    if norm == "keys":
        wq = None
    cache = new_cache(rt, g, kind, B, Hkv, cap, Dh, layers)
    pos = first + torch.randint(-3, 5000, (B, n), generator=g, device="cuda", dtype=torch.int32)
    L = [(7 * b) % 40 for b in range(B)]
    rows = rows or [n - (b % 2) * (n // 3) for b in range(B)]
    freq, _ = rt.rope_freqs(rot, 10000.0)
    out = q if in_place else torch.full((B, n, H, Dh), 3.0, dtype=DT[dtype], device="cuda")
    q0, out0, was = q.clone(), out.clone(), copies(cache)
    got = rt.norm_rope_append(q, k, v, pos, i32(L), i32(rows), freq, cache, q_norm=wq, k_norm=wk, eps=eps, layout=layout,
                              gain=gain, out=out)
    assert got is out
    (tq, lq), (tk, lk) = made(q0, wq, eps, pos, freq, gain, layout), made(k, wk, eps, pos, freq, gain, layout)
    for b in range(B):
        m, l = rows[b], L[b]
        assert torch.all((out[b, :m].double() - tq[b, :m]).abs() <= STEP[dtype] * tq[b, :m].abs() + 2.0 ** -20 * lq[b, :m])
        assert torch.equal(bits(out[b, m:]), bits(out0[b, m:]))
        m = max(0, min(m, cap - l))
        rest_same(parts(cache), was, b, slice(l, l + m))
        ks, vs = (t[b, :m].transpose(0, 1) for t in (tk, v))
        if kind in TOP:
            for t, codes, scale in ((ks, cache.k, cache.k_scale), (vs.double(), cache.v, cache.v_scale)):
                want, by = codes_of(t, kind)
                got_s = scale[b, :, l: l + m]
                assert torch.equal(torch.nan_to_num(got_s, nan=-1.0), torch.nan_to_num(by, nan=-1.0))
                assert torch.equal(codes[b, :, l: l + m].float(), want.float())
        else:
            got_k = cache.k[b, :, l: l + m].double()
            assert torch.all((got_k - ks).abs() <= STEP[dtype] * ks.abs() + 2.0 ** -48)
            assert torch.equal(bits(cache.v[b, :, l: l + m]), bits(vs))
    return cache


SHAPES = [
    (1, 1, 32, 32, 128, 128),
    (3, 61, 20, 20, 64, 64),
    (2, 5, 32, 8, 128, 64),       # grouped heads, half of each head
    (2, 17, 3, 1, 96, 22),        # pairs that no 16 bytes hold: one value at a time
    (2, 6, 4, 2, 96, 96),         # heads that are no power of two
    (1, 700, 4, 2, 64, 48),       # more rows than a tree
    (5, 2, 1, 1, 2, 2),           # the smallest head
    (1, 9, 2, 2, 256, 256),       # the largest
]


@pytest.mark.parametrize("kind", ["own", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_append(rt, dtype, kind, layout, shape):
    print(f"append {dtype} {kind} {layout} {shape}", flush=True)
    kind = dtype if kind == "own" else kind
    append_case(rt, dtype, kind, "shared", layout, *shape)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("norm", ["heads", "none", "keys"])
def test_append_norms(rt, kind, norm):
    print(f"append norms {kind} {norm}", flush=True)
    append_case(rt, "bf16", kind, norm, "half", 2, 9, 6, 2, 64, 64, gain=1.25, eps=0.5)
    append_case(rt, "bf16", kind, norm, "interleaved", 2, 9, 6, 2, 30, 8, gain=0.75)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_far_positions(rt, dtype):
    print(f"append far {dtype}", flush=True)
    append_case(rt, dtype, dtype, "shared", "half", 1, 33, 4, 4, 128, 128, first=1 << 20)


@pytest.mark.parametrize("kind", ["f32", "e4m3", "int8"])
def test_append_places(rt, kind):
    """In place, apart, layers of a larger cache, odd strides, a cache that is too short, no rows."""
    print(f"append places {kind}", flush=True)
    append_case(rt, "f32", kind, "shared", "half", 2, 5, 4, 4, 64, 64, fused=False, in_place=True)
    append_case(rt, "f32", kind, "shared", "interleaved", 2, 5, 4, 4, 54, 20, fused=False, in_place=True)
    append_case(rt, "f32", kind, "shared", "half", 3, 5, 4, 2, 64, 64, layers=3)
    append_case(rt, "f32", kind, "shared", "half", 3, 5, 4, 2, 64, 64, cap=17)       # ends within the third sequence's rows
    append_case(rt, "f32", kind, "shared", "half", 3, 5, 4, 2, 64, 64, rows=[0, 5, 0])


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("wide", [True, False])
def test_append_odd_rows(rt, kind, wide):
    """Rows of zeros, of values that are not finite, of the smallest and largest sizes, and halfway cases."""
    print(f"append odd {kind} {wide}", flush=True)
    Dh = 64 if wide else 62

    def edit(k, v):
        v[0, 0] = 0.0
        v[0, 1, 0, 5] = math.nan
        v[0, 2, 1, Dh - 1] = math.inf
        v[0, 3, 0, 0] = -math.inf
        v[0, 4] = 3e38
        v[0, 4, 0, 1] = -3.4e38
        v[0, 5] = v[0, 5] * 2.0 ** -145        # a few of the smallest steps: their scale is far off
        v[0, 6] = 2.0 ** -149                  # its scale rounds to 0
        v[0, 7] = torch.arange(Dh, device="cuda") + 0.5
        v[0, 7, :, 0] = TOP[kind]              # scale 1: codes halfway between two
        k[0, 8] = 0.0
        k[0, 9, 1, 3] = math.nan

    append_case(rt, "f32", kind, "shared", "half", 1, 11, 2, 2, Dh, Dh, edit=edit)
    append_case(rt, "f32", kind, "none", "half", 1, 11, 2, 2, Dh, Dh, edit=edit)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_append_many_rows(rt, layout):
    """Enough rows for several of them to a workgroup: ragged, past the cache's end, of sizes whose squares leave
    fp32, and sequences of two rows."""
    print(f"append many {layout}", flush=True)

    def edit(k, v):
        k[0, 5] *= 2.0 ** 100
        k[0, 6] *= 2.0 ** -100

    for dtype, kind, norm in (("bf16", "int8", "heads"), ("bf16", "bf16", "shared"), ("f32", "e4m3", "shared"), ("f32", "f32", "none")):
        append_case(rt, dtype, kind, norm, layout, 3, 703, 6, 2, 64, 48, cap=690, rows=[703, 2, 650], edit=edit)
        append_case(rt, dtype, kind, norm, layout, 1, 2049, 4, 4, 30, 10)
    append_case(rt, "bf16", "e4m3", "shared", layout, 1100, 2, 2, 1, 64, 64)


@pytest.mark.parametrize("dtype,kind", [("bf16", "int8"), ("bf16", "e4m3"), ("f32", "f32")])
def test_append_many_single_rows(rt, dtype, kind):
    """A decoding step of many sequences: one row each, some with none, caches that are full."""
    print(f"append single {dtype} {kind}", flush=True)
    append_case(rt, dtype, kind, "shared", "half", 1600, 1, 2, 1, 64, 64, rows=[int(b % 5 > 0) for b in range(1600)])
    append_case(rt, dtype, kind, "heads", "interleaved", 1537, 3, 2, 1, 64, 32, cap=4, rows=[b % 4 for b in range(1537)])


def test_append_large_queries(rt):
    """Queries whose squares leave fp32."""
    g = gen(12)
    q, kv = 2.0 ** 90 * normal(g, "f32", 1, 3, 4, 64), normal(g, "f32", 1, 3, 4, 64)
    cache = new_cache(rt, g, "f32", 1, 4, 8, 64)
    freq, _ = rt.rope_freqs(64)
    pos, w = i32([[5, 6, 7]]), torch.ones(64, device="cuda")
    out = rt.norm_rope_append(q, kv, kv, pos, i32([0]), i32([3]), freq, cache, q_norm=w)
    want, length = made(q, w, float(np.float32(1e-5)), pos, freq, 1.0, "half")
    assert torch.all((out.double() - want).abs() <= STEP["f32"] * want.abs() + 2.0 ** -20 * length)


def expect_queries(out, want, length, dtype):
    """Queries are the formula's to the roundings counted above; past the type's largest value they are infinite.  Below the
    smallest normal value, 2^-126, a rounding is off by half the smallest step whatever the size: 2^-134 the output's in
    bf16; 2^-150 each of up to 16 in fp32, which gains of up to 3 and two terms of a pair carry on: 2^-143."""
    least = (2.0 ** -134 if dtype == "bf16" else 0.0) + 2.0 ** -143
    most = torch.finfo(DT[dtype]).max
    got = out.double()
    past = want.abs() > 1.01 * most
    assert torch.equal(got[past], torch.sign(want[past]) * math.inf)
    inside = want.abs() < 0.99 * most
    assert torch.all(((got - want).abs() <= STEP[dtype] * want.abs() + 2.0 ** -20 * length + least)[inside])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Dh,rot", [(1, 64, 48), (2, 30, 10), (800, 64, 64)])
def test_append_queries_at_the_end_of_fp32(rt, dtype, layout, B, Dh, rot):
    """Squares, products with the gains and sums of pairs that leave fp32 where the normalised query does not,
    and pairs whose parts do where their sum does not: as they are, and among ordinary rows."""
    print(f"append ends {dtype} {layout} B={B} Dh={Dh}", flush=True)
    n, H, Hkv = 4, 3, 1
    g = gen(21)
    q = normal(g, "f32", B, n, H, Dh)
    sign = torch.where(q < 0, -1.0, 1.0)
    q[:, 0] = 3.3e38                                       # every pair's halves are the type's largest
    q[:, 1] = sign[:, 1] * 3.3e38 * torch.rand(B, H, Dh, device="cuda", generator=g)
    q[:, 2, 0] *= 2.0 ** 100                               # one head of an ordinary row
    q = q.to(DT[dtype])
    kv = normal(g, dtype, B, n, Hkv, Dh)
    pos = torch.randint(0, 5000, (B, n), generator=g, device="cuda", dtype=torch.int32)
    freq, _ = rt.rope_freqs(rot, 10000.0)
    eps, L, rows = float(np.float32(1e-5)), i32([0] * B), i32([n] * B)
    shared, heads = 1.0 + 2.0 * torch.rand(Dh, device="cuda", generator=g), 1.0 + torch.rand(H, Dh, device="cuda", generator=g)
    for w, gain in ((shared, 1.25), (heads, 0.75), (None, 1.0), (None, 2.0)):
        cache = new_cache(rt, g, dtype, B, Hkv, n, Dh)
        kn = None if w is None else torch.ones(Hkv, Dh, device="cuda") if w.dim() == 2 else w
        out = rt.norm_rope_append(q, kv, kv, pos, L, rows, freq, cache, q_norm=w, k_norm=kn, eps=eps, layout=layout, gain=gain)
        expect_queries(out, *made(q, w, eps, pos, freq, gain, layout), dtype)
    # small values of rows whose squares leave fp32
    few = 2.0 ** 66 * normal(g, dtype, B, n, H, Dh)
    few[..., 1::2] *= 2.0 ** -119                          # normalised some 2^-119, beside 1
    out = rt.norm_rope_append(few, kv, kv, pos, L, rows, freq, new_cache(rt, g, dtype, B, Hkv, n, Dh), q_norm=shared, eps=eps, layout=layout)
    expect_queries(out, *made(few, shared, eps, pos, freq, 1.0, layout), dtype)
    # gains so large that a value times them leaves fp32, and the row's factor brings it back
    w = torch.full((Dh,), 2.0 ** 70, device="cuda")
    q = 2.0 ** 60 * normal(g, dtype, B, n, H, Dh)
    out = rt.norm_rope_append(q, kv, kv, pos, L, rows, freq, cache, q_norm=w, eps=eps, layout=layout)
    expect_queries(out, *made(q, w, eps, pos, freq, 1.0, layout), dtype)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_small_queries_beside_large_ones(rt, dtype, layout):
    """A pair whose sum leaves fp32 changes nothing of the pairs beside it, however small they are."""
    print(f"append small beside large {dtype} {layout}", flush=True)
    for Dh, rot in ((64, 64), (128, 48), (30, 10)):
        g = gen(22)
        q = 1e-30 * (1.0 + torch.rand(1, 40, 4, Dh, device="cuda", generator=g))
        a, b = (0, rot // 2) if layout == "half" else (0, 1)
        q[..., a], q[..., b] = 3.3e38, -3.3e38
        q[0, ::5, :, Dh - 1] = math.inf
        q = q.to(DT[dtype])
        kv = normal(g, dtype, 1, 40, 1, Dh)
        pos = torch.arange(40, dtype=torch.int32, device="cuda")[None]
        freq, _ = rt.rope_freqs(rot)
        cache = new_cache(rt, g, dtype, 1, 1, 40, Dh)
        out = rt.norm_rope_append(q, kv, kv, pos, i32([0]), i32([40]), freq, cache, layout=layout, gain=1.5)
        finite = q.double()
        finite[torch.isinf(finite)] = 0.0
        want, length = made(finite, None, 0.0, pos, freq, 1.5, layout)
        keep = torch.ones(Dh, dtype=torch.bool, device="cuda")
        keep[[a, b, Dh - 1] + ([Dh // 2 - 1] if layout == "half" and rot == Dh else [Dh - 2])] = False      # (and the infinite ones' mates)
        expect_queries(out[..., keep], want[..., keep], length[..., keep], dtype)
        expect_queries(out[:, 1::5], want[:, 1::5], length[:, 1::5], dtype)


# ---------------------------------------------------------------------------- conversion
def convert_case(rt, dtype, kind, write, B, heads, Dh, cap, L, s0=None, d0=None, n_max=None, dcap=None, layers=0, seed=3, edit=None):
    g = gen(seed)
    src = new_cache(rt, g, dtype if write else kind, B, heads, cap, Dh, layers)
    dst = new_cache(rt, g, kind if write else dtype, B, heads, dcap or cap, Dh, layers)
    if edit:
        edit(src.k)
    was = copies(dst)
    got = rt.cache_convert(src, dst, i32(L), n_max, None if s0 is None else i32(s0), None if d0 is None else i32(d0))
    assert got is dst
    for b in range(B):
        f, t = (s0[b] if s0 else 0), (d0[b] if d0 else 0)
        n = max(0, min(L[b], n_max if n_max else L[b], cap - f, (dcap or cap) - t))
        lo = max(0, -f, -t)
        rest_same(parts(dst), was, b, slice(t + lo, t + n) if n > lo else slice(0, 0))
        if n <= lo:
            continue
        for x, xs, y, ys in ((src.k, src.k_scale, dst.k, dst.k_scale), (src.v, src.v_scale, dst.v, dst.v_scale)):
            x, y = x[b, :, f + lo: f + n], y[b, :, t + lo: t + n]
            if write:
                want, by = codes_of(x.double(), kind)
                assert torch.equal(y.float(), want.float())
                assert torch.equal(torch.nan_to_num(ys[b, :, t + lo: t + n], nan=-1.0), torch.nan_to_num(by, nan=-1.0))
            else:
                # an fp32 product, then the rounding to the type: as torch does them
                want = (x.float() * xs[b, :, f + lo: f + n, None]).to(DT[dtype])
                assert torch.equal(bits(y), bits(want))


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("write", [False, True])
@pytest.mark.parametrize("B,heads,Dh,cap,L", [
    (1, 8, 128, 700, [700]),
    (3, 2, 64, 100, [0, 1, 100]),
    (2, 3, 96, 50, [50, 33]),
    (2, 2, 256, 20, [20, 3]),
    (2, 2, 22, 70, [64, 70]),
    (4, 1, 2, 5, [5, 0, 2, 1]),
])
def test_convert(rt, dtype, kind, write, B, heads, Dh, cap, L):
    print(f"convert {dtype} {kind} write={write} B={B} heads={heads} Dh={Dh} cap={cap}", flush=True)
    convert_case(rt, dtype, kind, write, B, heads, Dh, cap, L)
    convert_case(rt, dtype, kind, write, B, heads, Dh, cap, L, layers=2)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("write", [False, True])
@pytest.mark.parametrize("Dh", [64, 30])
def test_convert_spans(rt, kind, write, Dh):
    """Starts on both sides, a bound below the lengths, caches of other lengths, and spans that leave them."""
    print(f"convert spans {kind} {write} {Dh}", flush=True)
    convert_case(rt, "bf16", kind, write, 3, 2, Dh, 90, [30, 0, 17], s0=[60, 5, 33], d0=[0, 3, 7], dcap=40)
    convert_case(rt, "bf16", kind, write, 2, 2, Dh, 90, [30, 17], s0=[1, 2], n_max=16)
    convert_case(rt, "bf16", kind, write, 5, 2, Dh, 90, [90, 50, 30, 40, 9], s0=[70, 0, -4, 95, 0], d0=[0, 20, 0, 0, -9], dcap=40, n_max=90)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_convert_odd_values(rt, kind):
    """Every bf16 value there is, NaN and infinities among them, and every code."""
    print(f"convert odd {kind}", flush=True)
    every = torch.arange(1 << 16, device="cuda").to(torch.int16).view(torch.bfloat16).view(1, 4, 256, 64)

    def edit(k):
        k.copy_(every)

    convert_case(rt, "bf16", kind, True, 1, 4, 64, 256, [256], edit=edit)

    def codes(k):
        k.view(torch.int8).copy_(torch.arange(4 * 256 * 64, device="cuda").to(torch.int8).view(1, 4, 256, 64))

    g = gen(5)
    src, dst = new_cache(rt, g, kind, 1, 4, 256, 64), new_cache(rt, g, "f32", 1, 4, 256, 64)
    codes(src.k)
    rt.cache_convert(src, dst, i32([256]))
    want = src.k.float() * src.k_scale[..., None]
    assert torch.equal(torch.isnan(dst.k), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(dst.k), torch.nan_to_num(want))


# ---------------------------------------------------------------------------- accepted paths
@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3", "int8"])
@pytest.mark.parametrize("B,slices,Dh,cap,n,a_max", [
    (1, 40, 128, 300, 61, 12), (3, 7, 64, 200, 128, 127), (2, 3, 256, 150, 17, 5), (2, 1, 32, 140, 9, 8), (4, 300, 64, 90, 12, 1),
])
def test_compact(rt, kind, B, slices, Dh, cap, n, a_max):
    print(f"compact {kind} B={B} slices={slices} Dh={Dh} cap={cap} n={n} a_max={a_max}", flush=True)
    for layers in (0, 3):
        g, rng = gen(4), np.random.default_rng(4)
        cache = new_cache(rt, g, kind, B, slices, cap, Dh, layers)
        L = [(11 * b) % (cap - n) for b in range(B)]
        n_acc = [a_max if b % 3 == 0 else int(rng.integers(0, a_max + 1)) for b in range(B)]
        path = np.zeros((B, a_max + 3), dtype=np.int32)
        for b in range(B):
            path[b, 1: a_max + 1] = np.sort(rng.choice(np.arange(1, n), size=a_max, replace=False))
        was = copies(cache)
        rt.cache_compact(cache, i32(L), torch.from_numpy(path).cuda(), i32(n_acc), a_max)
        for b in range(B):
            a = n_acc[b]
            rest_same(parts(cache), was, b, slice(L[b] + 1, L[b] + 1 + a))
            src = [L[b] + int(p) for p in path[b, 1: a + 1]]
            for x, y in zip(parts(cache), was):
                assert torch.equal(bits(x[b])[:, L[b] + 1: L[b] + 1 + a], bits(y[b])[:, src])


@pytest.mark.parametrize("kind,Dh,n,a_max", [("f32", 128, 128, 127), ("f32", 128, 100, 65), ("f32", 256, 128, 127), ("f32", 256, 60, 33),
                                             ("bf16", 256, 128, 127), ("bf16", 256, 128, 65)])
def test_compact_long_paths(rt, kind, Dh, n, a_max):
    """Paths of so many 16-byte pieces that a thread moves up to 32 of them."""
    assert a_max * Dh * DT[kind].itemsize // 16 > 2048
    test_compact(rt, kind, 3, 5, Dh, 300, n, a_max)


def test_compact_leaves_what_is_outside(rt):
    """Slots past the cache and path entries outside the tree stay where they are."""
    g = gen(6)
    cache = new_cache(rt, g, "int8", 2, 3, 20, 64)
    was = copies(cache)
    path = i32([[0, 2, 5, 9], [0, 0, -7, 500]])
    rt.cache_compact(cache, i32([14, 3]), path, i32([3, 3]), 3)
    rest_same(parts(cache), was, 1, slice(0, 0))
    rest_same(parts(cache), was, 0, slice(15, 17))
    for x, y in zip(parts(cache), was):
        assert torch.equal(bits(x[0])[:, 15:17], bits(y[0])[:, [16, 19]])


def test_caches_past_32_bits(rt):
    """Slots, heads and sequences whose elements lie past 2^31: append, conversion and a path there."""
    g = gen(8)
    cap, B, heads, Dh = 4_200_000, 2, 2, 256           # 2^31 codes in each sequence
    k, v = (torch.zeros(B, heads, cap, Dh, dtype=torch.int8, device="cuda") for _ in range(2))
    scales = [torch.zeros(B, heads, cap, device="cuda") for _ in range(2)]
    cache = rt.KVCache(k, v, *scales)
    L = [cap - 9, cap - 8]
    x, y = normal(g, "bf16", B, 8, heads, Dh), normal(g, "bf16", B, 8, heads, Dh)
    freq, _ = rt.rope_freqs(Dh)
    rt.norm_rope_append(x, x, y, torch.zeros(B, 8, dtype=torch.int32, device="cuda"), i32(L), i32([8, 8]), freq, cache)
    for t, codes, scale in ((x, k, scales[0]), (y, v, scales[1])):
        for b in range(B):
            want, by = codes_of(t[b].transpose(0, 1).double(), "int8")
            assert torch.equal(codes[b, :, L[b]: L[b] + 8].float(), want.float()) and torch.equal(scale[b, :, L[b]: L[b] + 8], by)
            assert not scale[b, :, L[b] - 3: L[b]].any()
    want = k[:, :, cap - 9:].clone()
    rt.cache_compact(cache, i32([cap - 9, cap - 9]), i32([[0, 3, 7]] * 2), i32([2, 2]), 2)
    assert torch.equal(k[:, :, cap - 8], want[:, :, 4 - 1]) and torch.equal(k[:, :, cap - 7], want[:, :, 7])
    window = new_cache(rt, g, "bf16", B, heads, 9, Dh)
    rt.cache_convert(cache, window, i32([9, 9]), src_start=i32([cap - 9] * 2))
    assert torch.equal(bits(window.k), bits((k[:, :, cap - 9:].float() * scales[0][:, :, cap - 9:, None]).bfloat16()))


@pytest.mark.parametrize("kind", ["int8", "bf16"])
def test_slots_of_a_head_past_32_bits(rt, kind):
    """Slots of one head whose elements lie past 2^31: append, conversion either way and a path there."""
    g = gen(10)
    cap, Dh = 8_400_000, 256                             # 2.15e9 elements a head
    caches = {k: rt.KVCache.zeros(1, 1, cap, Dh, DT[k]) for k in ("int8", "bf16")}
    cache, other = caches[kind], caches["bf16" if kind == "int8" else "int8"]
    L = cap - 9
    x, y = normal(g, "bf16", 1, 8, 1, Dh), normal(g, "bf16", 1, 8, 1, Dh)
    freq, _ = rt.rope_freqs(Dh)
    print(f"far slots {kind}", flush=True)
    rt.norm_rope_append(x, x, y, torch.zeros(1, 8, dtype=torch.int32, device="cuda"), i32([L]), i32([8]), freq, cache)
    for t, c, scale in ((x, cache.k, cache.k_scale), (y, cache.v, cache.v_scale)):
        rows = t[0].transpose(0, 1)
        if kind == "int8":
            want, by = codes_of(rows.double(), "int8")
            assert torch.equal(c[0, :, L: L + 8].float(), want.float()) and torch.equal(scale[0, :, L: L + 8], by)
        else:
            assert torch.equal(bits(c[0, :, L: L + 8]), bits(rows))
        assert not c[0, :, L - 3: L].any() and not c[0, :, L + 8:].any() and not c[0, :, :8].any()
    was = cache.v[:, :, L:].clone()
    rt.cache_compact(cache, i32([L]), i32([[0, 3, 7]]), i32([2]), 2)
    assert torch.equal(cache.v[:, :, L + 1], was[:, :, 3]) and torch.equal(cache.v[:, :, L + 2], was[:, :, 7])
    rt.cache_convert(cache, other, i32([9]), 9, i32([L]), i32([L]))
    for c, d, cs, ds in ((cache.k, other.k, cache.k_scale, other.k_scale), (cache.v, other.v, cache.v_scale, other.v_scale)):
        if kind == "int8":
            assert torch.equal(bits(d[:, :, L:]), bits((c[:, :, L:].float() * cs[:, :, L:, None]).bfloat16()))
        else:
            want, by = codes_of(c[:, :, L:].double(), "int8")
            assert torch.equal(d[:, :, L:].float(), want.float()) and torch.equal(ds[:, :, L:], by)
        assert not d[:, :, :9].any() and not d[:, :, L - 3: L].any()


def test_python_checks(rt):
    g = gen(9)
    c8, cb = new_cache(rt, g, "e4m3", 2, 2, 20, 64), new_cache(rt, g, "bf16", 2, 2, 20, 64)
    for bad in [lambda: rt.KVCache(c8.k, c8.v), lambda: rt.KVCache(cb.k, cb.v, c8.k_scale, c8.v_scale),
                lambda: rt.KVCache(c8.k, c8.v, c8.k_scale, None), lambda: rt.KVCache(c8.k, cb.v, c8.k_scale, c8.v_scale),
                lambda: rt.KVCache(c8.k.transpose(1, 2), c8.v.transpose(1, 2), c8.k_scale, c8.v_scale),
                lambda: rt.KVCache(c8.k, c8.v, c8.k_scale.double(), c8.v_scale),
                lambda: rt.KVCache(c8.k, c8.v, c8.k_scale[:, :, :10], c8.v_scale),
                lambda: rt.KVCache(cb.k.half(), cb.v.half()), lambda: rt.KVCache(cb.k.cpu(), cb.v.cpu())]:
        with pytest.raises(ValueError):
            bad()
    q, kv = normal(g, "bf16", 2, 3, 4, 64), normal(g, "bf16", 2, 3, 2, 64)
    pos, n = torch.zeros(2, 3, dtype=torch.int32, device="cuda"), i32([3, 3])
    freq, _ = rt.rope_freqs(64)
    ok = dict(q=q, k=kv, v=kv, pos=pos, kv_len=n, n_rows=n, freq=freq, cache=c8)
    one, two = torch.ones(64, device="cuda"), torch.ones(2, 64, device="cuda")
    for changed in [dict(q_norm=one.half()), dict(q_norm=two), dict(k_norm=one[:32]), dict(q_norm=one, k_norm=two), dict(k=q),
                    dict(pos=pos.long()), dict(kv_len=n[:1]), dict(freq=freq.float()), dict(v=kv.float())]:
        with pytest.raises(ValueError):
            rt.norm_rope_append(**{**ok, **changed})
    for args in [(c8, cb, n.long()), (c8, cb, n[:1])]:
        with pytest.raises(ValueError):
            rt.cache_convert(*args)
    from paper_2512_21857_amd.abi import AdtError
    for args in [(c8, c8, n), (cb, cb, n)]:
        with pytest.raises(AdtError):
            rt.cache_convert(*args)
