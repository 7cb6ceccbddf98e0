"""The operators over caches of any type on the CPU: refusals, each before anything is launched."""
import ctypes as C
import math

import pytest

FAKE = 0x100000


@pytest.fixture(scope="module")
def L():
    from paper_2512_21857_amd import abi
    return abi.lib()


def cache(at=FAKE, **changed):
    """A valid cache of two sequences of two heads, 100 slots of 64, in e4m3, with some fields changed."""
    from paper_2512_21857_amd import abi
    f = dict(k=at, v=at + 0x100000, stride_b=2 * 6400, stride_h=6400, k_scale=at + 0x200000, v_scale=at + 0x300000, scale_b=200,
             scale_h=100, B=2, heads=2, cap=100, Dh=64, type=abi.E4M3)
    assert set(changed) <= set(f)
    return abi.KvCache(*{**f, **changed}.values())


def plain(at=FAKE, **changed):
    return cache(at, **{**dict(k_scale=None, v_scale=None, type=1), **changed})


def call(fn, args, **changed):
    assert set(changed) <= set(args)
    args = {**args, **changed}
    return fn(*[C.byref(x) if isinstance(x, C.Structure) else x for x in args.values()])


CACHE = [
    (dict(k=None), "E_ARG"), (dict(v=None), "E_ARG"), (dict(type=4), "E_ARG"), (dict(type=-1), "E_ARG"),
    (dict(k_scale=None), "E_ARG"), (dict(type=1), "E_ARG"), (dict(B=0), "E_ARG"), (dict(heads=0), "E_ARG"),
    (dict(cap=0), "E_ARG"), (dict(Dh=0), "E_ARG"), (dict(Dh=63), "E_SHAPE"), (dict(Dh=258, stride_h=25800, stride_b=51600), "E_SHAPE"),
    (dict(heads=32768, stride_b=32768 * 6400, scale_b=32768 * 100), "E_SHAPE"), (dict(B=65536), "E_SHAPE"),
    (dict(stride_h=6399), "E_SHAPE"), (dict(stride_b=6400), "E_SHAPE"), (dict(scale_h=99), "E_SHAPE"), (dict(scale_b=100), "E_SHAPE"),
    (dict(cap=0x7f000001, stride_h=0x7f000001 * 64, stride_b=0x7f000001 * 128, scale_h=0x7f000001, scale_b=0x7f000001 * 2), "E_CAPACITY"),
]
WRITTEN = [(dict(v=FAKE), "E_ARG"), (dict(v_scale=FAKE + 0x200000), "E_ARG")]

FAR = 0x10000000
APPEND = dict(q=FAR, k=FAR + 0x10000, v=FAR + 0x20000, ldq=256, ldk=128, ldv=128, q_norm=FAKE, k_norm=FAKE, per_head=0, eps=1e-5,
              pos=FAKE, kv_len=FAKE, n_rows=FAKE, freq=FAKE, gain=1.0, rot=64, layout=0, n_max=3, H=4, dtype=1, q_out=FAR + 0x30000,
              cache=None, stream=None)


@pytest.mark.parametrize("changed,code", [
    (dict(q=None), "E_ARG"), (dict(freq=None), "E_ARG"), (dict(n_rows=None), "E_ARG"), (dict(q_out=None), "E_ARG"),
    (dict(dtype=2), "E_ARG"), (dict(layout=2), "E_ARG"), (dict(n_max=0), "E_ARG"), (dict(H=0), "E_ARG"), (dict(per_head=2), "E_ARG"),
    (dict(gain=math.inf), "E_ARG"), (dict(eps=0.0), "E_ARG"), (dict(eps=math.nan), "E_ARG"), (dict(eps=1e-39), "E_ARG"), (dict(rot=66), "E_SHAPE"),
    (dict(rot=0), "E_SHAPE"), (dict(rot=33), "E_SHAPE"), (dict(ldq=255), "E_SHAPE"), (dict(ldk=127), "E_SHAPE"),
    (dict(ldv=127), "E_SHAPE"), (dict(q_out=FAR, ldq=512), "E_SHAPE"), (dict(q_out=FAR + 16), "E_ARG"),
    (dict(q_out=FAR + 0x10000), "E_ARG"), (dict(q_out=FAR + 0x20000 - 16), "E_ARG"), (dict(H=1 << 20, ldq=64 << 20), "E_SHAPE"),
])
def test_norm_rope_append_refusals(L, changed, code):
    from paper_2512_21857_amd import abi
    assert call(L.adt_norm_rope_append, {**APPEND, "cache": cache()}, **changed) == getattr(abi, code), changed
    assert "norm_rope_append" in abi.last_error()


@pytest.mark.parametrize("changed,code", CACHE + WRITTEN)
def test_norm_rope_append_refuses_caches(L, changed, code):
    from paper_2512_21857_amd import abi
    assert call(L.adt_norm_rope_append, {**APPEND, "cache": cache(**changed)}) == getattr(abi, code), changed
    assert call(L.adt_norm_rope_append, APPEND) == abi.E_ARG


def test_norm_rope_append_refuses_other_plain_types(L):
    from paper_2512_21857_amd import abi
    assert call(L.adt_norm_rope_append, {**APPEND, "cache": plain(type=0)}) == abi.E_UNSUPPORTED
    assert call(L.adt_norm_rope_append, {**APPEND, "cache": plain(), "dtype": 0}) == abi.E_UNSUPPORTED


CONVERT = dict(src=None, dst=None, length=FAKE, n_max=100, src_start=None, dst_start=None, stream=None)


@pytest.mark.parametrize("changed,code", CACHE)
def test_cache_convert_refuses_caches(L, changed, code):
    from paper_2512_21857_amd import abi
    fn = L.adt_cache_convert
    assert call(fn, {**CONVERT, "src": cache(**changed), "dst": plain(FAR)}) == getattr(abi, code), changed
    assert call(fn, {**CONVERT, "src": plain(FAR), "dst": cache(**changed)}) == getattr(abi, code), changed
    assert "cache_convert" in abi.last_error()


def test_cache_convert_refusals(L):
    from paper_2512_21857_amd import abi
    ok = {**CONVERT, "src": cache(), "dst": plain(FAR)}
    for changed, code in [
        (dict(length=None), abi.E_ARG), (dict(n_max=0), abi.E_ARG), (dict(n_max=0x7f000001), abi.E_CAPACITY),
        (dict(src=None), abi.E_ARG), (dict(dst=None), abi.E_ARG), (dict(dst=cache(FAR)), abi.E_UNSUPPORTED),
        (dict(src=plain()), abi.E_UNSUPPORTED), (dict(dst=plain(FAR, type=0), src=plain()), abi.E_UNSUPPORTED),
        (dict(dst=plain(FAR, B=1)), abi.E_SHAPE), (dict(dst=plain(FAR, heads=1)), abi.E_SHAPE),
        (dict(dst=plain(FAR, Dh=32)), abi.E_SHAPE), (dict(dst=plain(FAR, v=FAR)), abi.E_ARG),
        # 25600 bytes of codes from FAKE on, 51200 of values
        (dict(dst=plain(FAKE + 25584)), abi.E_ARG), (dict(dst=plain(FAR, v=FAKE - 51184)), abi.E_ARG),
    ]:
        assert call(L.adt_cache_convert, ok, **changed) == code, changed


@pytest.mark.parametrize("scales", ["k_scale", "v_scale"])
def test_cache_convert_refuses_scales_among_values(L, scales):
    """1600 bytes of scales, 51200 of values: neither direction may write one while reading the other."""
    from paper_2512_21857_amd import abi
    for at in (FAR - 1584, FAR, FAR + 51184):
        codes = cache(**{scales: at})
        assert call(L.adt_cache_convert, {**CONVERT, "src": codes, "dst": plain(FAR)}) == abi.E_ARG, hex(at)
        assert call(L.adt_cache_convert, {**CONVERT, "src": plain(FAR), "dst": codes}) == abi.E_ARG, hex(at)
    assert "overlap" in abi.last_error()


COMPACT = dict(cache=None, kv_len=FAKE, path=FAKE, stride=9, n_acc=FAKE, a_max=8, stream=None)


@pytest.mark.parametrize("changed,code", CACHE + WRITTEN + [
    (dict(k=FAKE + 8), "E_SHAPE"), (dict(stride_h=6408, stride_b=2 * 6408), "E_SHAPE"), (dict(Dh=40), "E_SHAPE"),
])
def test_cache_compact_refuses_caches(L, changed, code):
    from paper_2512_21857_amd import abi
    assert call(L.adt_cache_compact, {**COMPACT, "cache": cache(**changed)}) == getattr(abi, code), changed
    assert "cache_compact" in abi.last_error()


@pytest.mark.parametrize("changed,code", [
    (dict(kv_len=None), "E_ARG"), (dict(path=None), "E_ARG"), (dict(n_acc=None), "E_ARG"), (dict(a_max=-1), "E_CAPACITY"),
    (dict(a_max=128, stride=200), "E_CAPACITY"), (dict(stride=8), "E_CAPACITY"),
])
def test_cache_compact_refusals(L, changed, code):
    from paper_2512_21857_amd import abi
    assert call(L.adt_cache_compact, {**COMPACT, "cache": cache()}, **changed) == getattr(abi, code), changed
    assert call(L.adt_cache_compact, {**COMPACT, "cache": cache(), "a_max": 0}) == abi.OK


ATTN = dict(q=FAKE, cache=None, kv_len=FAKE, n_q=FAKE, n_tail=FAKE, mask=FAKE, H=4, nq_max=8, kv_cap=100, prefix=None,
            prefix_len=None, prefix_cap=0, scale=0.125, dtype=1, out=FAR, ws=FAKE, ws_bytes=1 << 40, stream=None)


def behind(**changed):
    return {**ATTN, "cache": cache(), "prefix": cache(B=1, **changed), "prefix_len": FAKE, "prefix_cap": 100}


@pytest.mark.parametrize("changed,code", CACHE + [
    (dict(k=FAKE + 8), "E_SHAPE"), (dict(stride_h=6408, stride_b=2 * 6408), "E_SHAPE"), (dict(Dh=32), "E_SHAPE"),
    (dict(cap=99), "E_CAPACITY"),
])
def test_cache_tree_attn_refuses_caches(L, changed, code):
    from paper_2512_21857_amd import abi
    assert call(L.adt_cache_tree_attn, {**ATTN, "cache": cache(**changed)}) == getattr(abi, code), changed
    assert "cache_tree_attn" in abi.last_error()


@pytest.mark.parametrize("changed,code", [
    (dict(q=None), "E_ARG"), (dict(mask=None), "E_ARG"), (dict(n_tail=None), "E_ARG"), (dict(out=None), "E_ARG"),
    (dict(prefix_len=None), "E_ARG"), (dict(dtype=3), "E_ARG"), (dict(dtype=0), "E_UNSUPPORTED"), (dict(H=0), "E_ARG"),
    (dict(H=5), "E_SHAPE"), (dict(kv_cap=0), "E_ARG"), (dict(kv_cap=101), "E_CAPACITY"), (dict(prefix_cap=101), "E_CAPACITY"),
    (dict(prefix_cap=0), "E_ARG"), (dict(nq_max=0), "E_CAPACITY"), (dict(nq_max=129), "E_CAPACITY"),
    (dict(nq_max=128, H=256), "E_CAPACITY"), (dict(scale=0.0), "E_ARG"), (dict(scale=math.nan), "E_ARG"), (dict(out=FAKE + 16), "E_ARG"),
    (dict(out=FAR + 8), "E_SHAPE"), (dict(q=FAKE + 2), "E_SHAPE"), (dict(ws=FAKE + 4), "E_SHAPE"), (dict(ws=None), "E_CAPACITY"),
    (dict(ws_bytes=64), "E_CAPACITY"),
])
def test_cache_tree_attn_refusals(L, changed, code):
    from paper_2512_21857_amd import abi
    assert call(L.adt_cache_tree_attn, behind(), **changed) == getattr(abi, code), changed
    assert "cache_tree_attn" in abi.last_error()


def test_cache_tree_attn_refuses_prefixes(L):
    from paper_2512_21857_amd import abi
    for changed, code in [(dict(type=3), abi.E_UNSUPPORTED), (dict(heads=1), abi.E_SHAPE), (dict(Dh=32), abi.E_SHAPE),
                          (dict(k=None), abi.E_ARG), (dict(k=FAKE + 8), abi.E_SHAPE), (dict(cap=99), abi.E_CAPACITY)]:
        assert call(L.adt_cache_tree_attn, behind(**changed)) == code, changed
    a = behind()
    assert call(L.adt_cache_tree_attn, {**a, "cache": cache(B=3), "prefix": cache()}) == abi.E_SHAPE
    many = dict(B=4097, heads=1, stride_b=6400, scale_b=100)
    assert call(L.adt_cache_tree_attn, {**a, "cache": cache(**many), "prefix": cache(B=1, heads=1)}) == abi.E_CAPACITY
    assert call(L.adt_cache_tree_attn, {**a, "cache": plain(type=0), "prefix": plain(B=1, type=0)}) == abi.E_UNSUPPORTED


def test_cache_tree_attn_workspace_sizes(L):
    size = L.adt_cache_tree_attn_workspace_size
    ok = (16, 32, 8, 128, 61, 4096, 2, 2048, 2)
    assert size(*ok) > 0
    for i, bad in [(0, 0), (0, 65536), (1, 33), (2, 0), (3, 96), (4, 129), (4, 0), (5, 0), (5, 0x7f000001), (6, 3), (6, -1), (7, 0),
                   (7, 0x7f000001), (8, 4), (8, -1), (1, 1 << 30)]:
        assert size(*ok[:i], bad, *ok[i + 1:]) == 0, (i, bad)
    assert size(1, 4, 4, 64, 8, 64, 0, 0, 1) == 0              # keys of one job: nothing to merge
    assert size(8192, 7, 7, 64, 128, 64, 2, 64, 3) > 0 and size(8194, 7, 7, 64, 1, 64, 2, 64, 3) == 0   # 4096, 4097 a group
    # the largest sizes: so many pairs that their keys are not split, and many rows behind one prefix
    assert size(65535, 64, 1, 64, 128, 0x7f000000, 0, 0, 2) == 0
    assert 2 * 4096 * 15 * 8192 * 66 * 4 <= size(4096, 3840, 15, 64, 32, 0x7f000000, 1, 0x7f000000, 0) < 1 << 50


@pytest.mark.parametrize("B,H,heads,Dh,nq,kv_cap,groups,prefix_cap", [
    (1, 32, 8, 128, 1, 65536, 0, 0), (16, 32, 32, 128, 61, 2560, 1, 2112), (64, 32, 8, 128, 1, 576, 1, 32768),
    (4, 4, 4, 64, 17, 192, 2, 256), (2, 8, 1, 64, 40, 5000, 1, 300), (3, 6, 2, 128, 8, 30000, 3, 30000), (1, 1, 1, 64, 1, 0x7f000000, 1, 0x7f000000),
])
def test_cache_tree_attn_workspace_holds_for_smaller_bounds(L, B, H, heads, Dh, nq, kv_cap, groups, prefix_cap):
    """What is enough for some bounds is enough for every pair of smaller ones, and without the prefix."""
    size = L.adt_cache_tree_attn_workspace_size
    for kind in (0, 1, 2, 3):
        steps = lambda top: sorted({max(1, top * i // 40) for i in range(1, 41)} | {max(1, int(top / 1.3 ** i)) for i in range(60)})  # noqa: E731
        caps, pcaps = steps(kv_cap), steps(prefix_cap) if groups else [0]
        sizes = [[size(B, H, heads, Dh, nq, c, groups, p, kind) for p in pcaps] for c in caps]
        for i in range(len(caps)):
            for j in range(len(pcaps)):
                assert (i == 0 or sizes[i][j] >= sizes[i - 1][j]) and (j == 0 or sizes[i][j] >= sizes[i][j - 1]), (kind, caps[i], pcaps[j])
            assert not groups or sizes[i][0] >= size(B, H, heads, Dh, nq, caps[i], 0, 0, kind)


def test_python_cache_refusals():
    import torch
    from paper_2512_21857_amd import runtime as rt
    with pytest.raises(ValueError, match="device tensor"):
        rt.KVCache(torch.zeros(1, 1, 4, 64), torch.zeros(1, 1, 4, 64))
