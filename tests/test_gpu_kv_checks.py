"""Invariant checks of the debug build in the calls over caches of any type: lengths, starts and accepted
paths lie on the device, where the host cannot see them.  The kernels stay within the cache either way;
a debug build records the violation, which adt_device_check reports and clears, and the release build
records nothing."""
import ctypes as C

import pytest
import torch

pytestmark = pytest.mark.gpu

KINDS = [torch.bfloat16, torch.float32, torch.int8, torch.float8_e4m3fn]
B, HEADS, SLOTS, DH, NQ = 2, 2, 64, 64, 4


@pytest.fixture(scope="module")
def libs():
    from paper_2512_21857_amd import abi, runtime
    assert torch.cuda.is_available()
    return abi, runtime, abi.lib(), abi.lib_debug()


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def p(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def ref(cache):
    return None if cache is None else C.byref(cache._struct)


def bits(cache):
    return [t.clone().view(torch.uint8) for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None]


def cache_of(rt, kind, seed=3):
    """A cache of codes or values that are not zero, its rows all different."""
    c = rt.KVCache.zeros(B, HEADS, SLOTS, DH, kind)
    g = torch.Generator(device="cuda").manual_seed(seed)
    for t in (c.k, c.v):
        t.copy_(torch.randint(-60, 60, t.shape, generator=g, device="cuda").float().to(kind))
    for t in (c.k_scale, c.v_scale):
        if t is not None:
            t.uniform_(0.01, 0.02, generator=g)
    return c


def expect(libs, call, word):
    """call(L) breaks an invariant: the debug build says so, once, the release build does not."""
    abi, _, R, D = libs
    assert call(D) == 0
    assert D.adt_device_check(stream()) == abi.E_DEVICE_INVARIANT and word in abi.last_error(D)
    assert D.adt_device_check(stream()) == abi.OK
    assert call(R) == 0
    assert R.adt_device_check(stream()) == abi.OK


@pytest.mark.parametrize("kind", KINDS)
def test_append_past_the_cache(libs, kind):
    abi, rt, R, D = libs
    print(f"append {kind}", flush=True)
    dt = torch.float32 if kind == torch.float32 else torch.bfloat16
    q, k, v = (torch.ones(B, NQ, HEADS, DH, dtype=dt, device="cuda") for _ in range(3))
    freq, pos = torch.ones(DH // 2, dtype=torch.float64, device="cuda"), torch.zeros(B, NQ, dtype=torch.int32, device="cuda")
    out, c = torch.empty_like(q), cache_of(rt, kind)
    n = i32(NQ, 2)

    def run(L, *lens):
        kl = i32(*lens)
        return L.adt_norm_rope_append(p(q), p(k), p(v), HEADS * DH, HEADS * DH, HEADS * DH, None, None, 0, 1e-5, p(pos), p(kl),
                                      p(n), p(freq), 1.0, DH, 0, NQ, HEADS, abi.F32 if dt == torch.float32 else abi.BF16, p(out),
                                      ref(c), stream())

    before = bits(c)
    assert run(D, SLOTS - NQ, 0) == 0
    assert D.adt_device_check(stream()) == abi.OK
    c = cache_of(rt, kind)
    expect(libs, lambda L: run(L, SLOTS - 2, -1), "cache capacity")
    # two rows fit into sequence 0; a negative length has no slots
    for now, was in zip(bits(c), before):
        assert torch.equal(now[1], was[1]) and torch.equal(now[0, :, : SLOTS - 2], was[0, :, : SLOTS - 2])
        assert not torch.equal(now[0, :, SLOTS - 2:], was[0, :, SLOTS - 2:])


@pytest.mark.parametrize("kind", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("read", [False, True])
def test_convert_past_the_cache(libs, kind, read):
    abi, rt, R, D = libs
    print(f"convert {kind} read={read}", flush=True)
    src, dst = cache_of(rt, kind if read else torch.bfloat16), cache_of(rt, torch.bfloat16 if read else kind, seed=4)

    def run(L, lens, starts):
        n, s = i32(*lens), i32(*starts)
        return L.adt_cache_convert(ref(src), ref(dst), p(n), SLOTS, p(s), p(s), stream())

    assert run(D, (5, 0), (SLOTS - 5, 0)) == 0
    assert D.adt_device_check(stream()) == abi.OK
    before = bits(dst)
    expect(libs, lambda L: run(L, (6, 0), (SLOTS - 5, 0)), "cache capacity")
    expect(libs, lambda L: run(L, (0, 1), (0, -1)), "cache capacity")
    for now, was in zip(bits(dst), before):
        assert torch.equal(now, was)                         # (the rows inside are those of the first call)


@pytest.mark.parametrize("kind", KINDS)
def test_compact_outside_the_tree(libs, kind):
    abi, rt, R, D = libs
    print(f"compact {kind}", flush=True)
    c = cache_of(rt, kind)

    def run(L, path, kv_len=10):
        pt, n, kl = torch.tensor([path, [0, 1, 2, 3]], dtype=torch.int32, device="cuda"), i32(3, 0), i32(kv_len, 10)
        return L.adt_cache_compact(ref(c), p(kl), p(pt), 4, p(n), 3, stream())

    assert run(D, [0, 1, 3, 7]) == 0
    assert D.adt_device_check(stream()) == abi.OK
    before = bits(c)
    expect(libs, lambda L: run(L, [0, 1, 2, 999]), "accepted-path")
    expect(libs, lambda L: run(L, [0, 1, 2, -5]), "accepted-path")
    expect(libs, lambda L: run(L, [0, 1, 2, 40], SLOTS - 10), "cache capacity")
    for now, was in zip(bits(c), before):
        assert torch.equal(now, was)                         # no other row moved


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("own,pre", [(SLOTS, 0), (4, SLOTS + 9), (SLOTS + 9, 5)])
def test_attention_past_the_cache(libs, kind, own, pre):
    """Keys from the bounds on do not count; what a full cache gives is what is left."""
    abi, rt, R, D = libs
    print(f"attn {kind} own={own} prefix={pre}", flush=True)
    c, x = cache_of(rt, kind), cache_of(rt, kind, seed=5)
    dt = torch.float32 if kind == torch.float32 else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(6)
    q = torch.randn(B, NQ, HEADS, DH, generator=g, device="cuda").to(dt)
    mask = torch.zeros(B, NQ, 2, dtype=torch.int64, device="cuda")
    mask[:, :, 0] = 15
    n = i32(NQ, NQ)
    name = {torch.bfloat16: abi.BF16, torch.float32: abi.F32, torch.int8: abi.I8, torch.float8_e4m3fn: abi.E4M3}[kind]
    need = R.adt_cache_tree_attn_workspace_size(B, HEADS, HEADS, DH, NQ, SLOTS, B, SLOTS, name)
    ws = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")

    def run(L, own, pre, tail, out):
        kl, pl, t = i32(own, 3), i32(pre, 2), i32(tail, tail)
        return L.adt_cache_tree_attn(p(q), ref(c), p(kl), p(n), p(t), p(mask), HEADS, NQ, SLOTS, ref(x), p(pl), SLOTS, 0.125,
                                     abi.F32 if dt == torch.float32 else abi.BF16, p(out), p(ws), ws.numel(), stream())

    outs = [torch.empty_like(q) for _ in range(3)]
    left = min(NQ, max(0, SLOTS - own))                      # tail slots inside the cache
    n_full = i32(left, NQ)
    kl, pl = i32(min(own, SLOTS), 3), i32(min(pre, SLOTS), 2)
    assert D.adt_cache_tree_attn(p(q), ref(c), p(kl), p(n), p(n_full), p(mask), HEADS, NQ, SLOTS, ref(x), p(pl), SLOTS, 0.125,
                                 abi.F32 if dt == torch.float32 else abi.BF16, p(outs[0]), p(ws), ws.numel(), stream()) == 0
    assert D.adt_device_check(stream()) == abi.OK
    which = iter(outs[1:])
    expect(libs, lambda L: run(L, own, pre, NQ, next(which)), "cache capacity")
    for o in outs[1:]:
        assert torch.isfinite(o.float()).all() and torch.equal(o, outs[0])
