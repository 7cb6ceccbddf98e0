"""The operators of a long or bounded cache on the CPU: refusals, each before anything is
launched, and the host-only rotary frequencies against their formulas."""
import ctypes as C
import math
import subprocess
import sys

import numpy as np
import pytest

FAKE = 0x1000


@pytest.fixture(scope="module")
def L():
    from paper_2512_21857_amd import abi
    return abi.lib()


def call(fn, args, **changed):
    """fn with a valid argument list (an ordered dict) in which some entries are changed."""
    assert set(changed) <= set(args)
    return fn(*{**args, **changed}.values())


ROPE = dict(q=FAKE, k=FAKE, v=FAKE, ldq=256, ldk=128, ldv=128, pos=FAKE, kv_len=FAKE, n_rows=FAKE, freq=FAKE, gain=1.0,
            rot=64, layout=0, B=2, n_max=3, H=4, Hkv=2, Dh=64, q_out=FAKE + 16, kc=FAKE, vc=FAKE, sb=2 * 64 * 100,
            sh=64 * 100, cap=100, dtype=1, stream=None)


@pytest.mark.parametrize("changed,code", [
    (dict(q=None), "E_ARG"), (dict(freq=None), "E_ARG"), (dict(vc=None), "E_ARG"), (dict(dtype=2), "E_ARG"),
    (dict(layout=2), "E_ARG"), (dict(B=0), "E_ARG"), (dict(n_max=0), "E_ARG"), (dict(Hkv=0), "E_ARG"),
    (dict(gain=math.nan), "E_ARG"), (dict(Dh=63), "E_SHAPE"), (dict(Dh=258, rot=64), "E_SHAPE"), (dict(rot=66), "E_SHAPE"),
    (dict(rot=33), "E_SHAPE"), (dict(rot=0), "E_SHAPE"), (dict(ldq=255), "E_SHAPE"), (dict(ldv=127), "E_SHAPE"),
    (dict(q_out=FAKE, ldq=512), "E_SHAPE"), (dict(sh=64 * 99), "E_SHAPE"), (dict(sb=64 * 100), "E_SHAPE"),
])
def test_rope_append_refusals(L, changed, code):
    from paper_2512_21857_amd import abi
    assert call(L.adt_rope_append, ROPE, **changed) == getattr(abi, code), changed
    assert "rope_append" in abi.last_error()


def freqs(L, rot, scaling, theta=10000.0, factor=1.0, orig=4096, fast=32.0, slow=1.0):
    from paper_2512_21857_amd import abi
    cfg = abi.RopeCfg(rot, scaling, theta, factor, orig, fast, slow)
    f = (C.c_double * 128)()
    g = C.c_float()
    code = L.adt_rope_freqs(C.byref(cfg), f, C.byref(g))
    return code, np.array(f[: max(rot, 0) // 2]), g.value


def test_rope_freqs_formulas(L):
    from paper_2512_21857_amd import abi
    rot, theta, s = 64, 10000.0, 8.0
    i = np.arange(rot // 2)
    plain = theta ** (-2.0 * i / rot)
    for scaling, want in ((abi.ROPE_PLAIN, plain), (abi.ROPE_LINEAR, plain / s),
                          (abi.ROPE_BASE, (theta * s ** (rot / (rot - 2))) ** (-2.0 * i / rot))):
        code, f, g = freqs(L, rot, scaling, theta, s)
        assert code == abi.OK and g == 1.0
        np.testing.assert_allclose(f, want, rtol=1e-14)
    # the stretched base leaves the highest frequency and divides the lowest by the factor
    _, f, _ = freqs(L, rot, abi.ROPE_BASE, theta, s)
    assert f[0] == 1.0 and abs(f[-1] * s / plain[-1] - 1) < 1e-12
    code, f, g = freqs(L, rot, abi.ROPE_RAMP, theta, s, 4096)
    assert code == abi.OK and g == np.float32(0.1 * math.log(s) + 1)
    turns = 4096 * plain / (2 * math.pi)
    # well above 32 turns unchanged, well below one divided, in between monotone
    assert np.allclose(f[turns > 64], plain[turns > 64], rtol=1e-14) and np.allclose(f[turns < 0.5], plain[turns < 0.5] / s, rtol=1e-14)
    share = (1 - f / plain) / (1 - 1 / s)
    assert np.all(np.diff(share) > -1e-12) and 0.3 < share[np.argmin(abs(turns - math.sqrt(32)))] < 0.7
    # an original context so short that no frequency turns once: all of them divided but the first
    code, f, _ = freqs(L, rot, abi.ROPE_RAMP, theta, s, 1)
    assert code == abi.OK and np.allclose(f[1:], plain[1:] / s, rtol=1e-14)
    assert freqs(L, 2, abi.ROPE_BASE, theta, s)[1].tolist() == [1.0]


@pytest.mark.parametrize("kw,code", [
    (dict(rot=63), "E_SHAPE"), (dict(rot=0), "E_SHAPE"), (dict(rot=258), "E_SHAPE"), (dict(scaling=4), "E_ARG"),
    (dict(scaling=-1), "E_ARG"), (dict(theta=1.0), "E_ARG"), (dict(theta=math.inf), "E_ARG"),
    (dict(scaling=1, factor=0.5), "E_ARG"), (dict(scaling=2, factor=math.nan), "E_ARG"),
    (dict(scaling=3, factor=4.0, orig=0), "E_ARG"), (dict(scaling=3, factor=4.0, fast=1.0, slow=1.0), "E_ARG"),
    (dict(scaling=3, factor=4.0, slow=0.0), "E_ARG"),
])
def test_rope_freqs_refusals(L, kw, code):
    from paper_2512_21857_amd import abi
    kw = {"rot": 64, "scaling": 0, **kw}
    assert freqs(L, kw.pop("rot"), kw.pop("scaling"), **kw)[0] == getattr(abi, code)
    assert L.adt_rope_freqs(None, None, None) == abi.E_ARG


KEYS = dict(k=FAKE, sb=2 * 64 * 100, sh=64 * 100, start=None, kv_len=FAKE, B=2, Hkv=2, Dh=64, block=32, cap=100, means=FAKE,
            mb=2 * 64 * 4, mh=64 * 4, dtype=1, stream=None)


@pytest.mark.parametrize("changed,code", [
    (dict(k=None), "E_ARG"), (dict(kv_len=None), "E_ARG"), (dict(means=None), "E_ARG"), (dict(dtype=-1), "E_ARG"),
    (dict(B=0), "E_ARG"), (dict(Hkv=70000), "E_ARG"), (dict(Dh=96), "E_SHAPE"), (dict(block=48), "E_SHAPE"),
    (dict(block=0), "E_SHAPE"), (dict(block=16), "E_SHAPE"), (dict(sh=64 * 99), "E_SHAPE"), (dict(mh=64 * 3), "E_SHAPE"),
    (dict(sb=64), "E_SHAPE"), (dict(mb=64 * 4), "E_SHAPE"), (dict(k=FAKE + 8), "E_SHAPE"), (dict(means=FAKE + 4), "E_SHAPE"),
    (dict(sh=64 * 100 + 4, sb=4 * 64 * 100), "E_SHAPE"),
])
def test_block_keys_refusals(L, changed, code):
    from paper_2512_21857_amd import abi
    assert call(L.adt_block_keys, KEYS, **changed) == getattr(abi, code), changed
    assert "block_keys" in abi.last_error()


ATTN = dict(q=FAKE, k=FAKE, v=FAKE, sb=2 * 64 * 100, sh=64 * 100)
SIZES = dict(kv_len=FAKE, n_q=FAKE, n_tail=FAKE, mask=FAKE, B=2, H=4, Hkv=2, Dh=64, nq_max=8, cap=100)
SPARSE = {**ATTN, **dict(means=FAKE, mb=2 * 64 * 4, mh=64 * 4), **SIZES,
          **dict(block=32, n_sel=3, n_first=1, n_last=1, scale=0.125, dtype=1, out=FAKE, sel=None, ws=FAKE, ws_bytes=1 << 30,
                 stream=None)}
RATED = {**ATTN, **SIZES, **dict(scale=0.125, dtype=1, out=FAKE, w_in=None, w_out=FAKE, wb=200, wh=100, decay=1.0, rw=None,
                                 ws=FAKE, ws_bytes=1 << 30, stream=None)}
COMMON = [
    (dict(q=None), "E_ARG"), (dict(mask=None), "E_ARG"), (dict(n_tail=None), "E_ARG"), (dict(out=None), "E_ARG"),
    (dict(dtype=3), "E_ARG"), (dict(B=0), "E_ARG"), (dict(H=0), "E_ARG"), (dict(Hkv=0), "E_ARG"), (dict(H=5), "E_SHAPE"),
    (dict(Dh=96), "E_SHAPE"), (dict(nq_max=129), "E_CAPACITY"), (dict(nq_max=0), "E_CAPACITY"),
    (dict(nq_max=128, H=256, Hkv=2), "E_CAPACITY"), (dict(sh=64 * 99), "E_SHAPE"), (dict(sb=64 * 100), "E_SHAPE"),
    (dict(k=FAKE + 2), "E_SHAPE"), (dict(out=FAKE + 8), "E_SHAPE"), (dict(sh=64 * 100 + 4, sb=4 * 64 * 100), "E_SHAPE"),
    (dict(scale=0.0), "E_ARG"), (dict(scale=math.inf), "E_ARG"), (dict(ws=None), "E_CAPACITY"), (dict(ws=FAKE + 4), "E_SHAPE"),
    (dict(ws_bytes=64), "E_CAPACITY"),
]


@pytest.mark.parametrize("changed,code", COMMON + [
    (dict(means=None), "E_ARG"), (dict(block=16), "E_SHAPE"), (dict(n_sel=0), "E_ARG"), (dict(n_first=2, n_last=2), "E_ARG"),
    (dict(n_first=-1), "E_ARG"), (dict(mh=64 * 3), "E_SHAPE"), (dict(means=FAKE + 4), "E_SHAPE"),
    (dict(B=1, cap=16385 * 32, sh=64 * 16385 * 32, mh=64 * 16385), "E_CAPACITY"),
])
def test_sparse_tree_attn_refusals(L, changed, code):
    from paper_2512_21857_amd import abi
    assert call(L.adt_sparse_tree_attn, SPARSE, **changed) == getattr(abi, code), changed
    assert "sparse_tree_attn" in abi.last_error()


@pytest.mark.parametrize("changed,code", COMMON + [
    (dict(w_out=None), "E_ARG"), (dict(decay=math.nan), "E_ARG"), (dict(wh=99), "E_SHAPE"), (dict(wb=100), "E_SHAPE"),
])
def test_tree_attn_weights_refusals(L, changed, code):
    from paper_2512_21857_amd import abi
    assert call(L.adt_tree_attn_weights, RATED, **changed) == getattr(abi, code), changed
    assert "tree_attn_weights" in abi.last_error()


def test_outputs_over_the_queries(L):
    """Rated attention reads its queries again after the output is written, so the two may not share
    memory; over chosen blocks the output may be the queries, but not lie across them."""
    from paper_2512_21857_amd import abi
    q = 1 << 20
    size = SIZES["B"] * SIZES["nq_max"] * SIZES["H"] * SIZES["Dh"] * 2
    for out in (q, q + 16, q - 16, q + size - 16, q - size + 16):
        assert call(L.adt_tree_attn_weights, RATED, q=q, out=out) == abi.E_ARG, out - q
        assert "overlaps" in abi.last_error()
        if out != q:
            assert call(L.adt_sparse_tree_attn, SPARSE, q=q, out=out) == abi.E_ARG, out - q
            assert "overlaps" in abi.last_error()


def test_attention_workspaces(L):
    """Sizes for what the calls take, 0 for what they refuse."""
    sparse = lambda *a: L.adt_sparse_tree_attn_workspace_size(*a)       # noqa: E731
    rated = lambda *a: L.adt_tree_attn_weights_workspace_size(*a)       # noqa: E731
    assert sparse(1, 32, 8, 128, 61, 4096, 64, 16, 1) > 0 and rated(1, 32, 8, 128, 61, 4096, 1) > 0
    for bad in ((0, 32, 8, 128, 61, 4096), (1, 33, 8, 128, 61, 4096), (1, 32, 8, 96, 61, 4096), (1, 32, 8, 128, 129, 4096),
                (1, 32, 8, 128, 61, 0)):
        assert sparse(*bad, 64, 16, 1) == 0 and rated(*bad, 1) == 0
    assert sparse(1, 32, 8, 128, 61, 4096, 48, 16, 1) == 0 and sparse(1, 32, 8, 128, 61, 4096, 64, 0, 1) == 0
    assert rated(1, 32, 8, 128, 61, 4096, 2) == 0


@pytest.mark.parametrize("B,H,Hkv,nq_max", [
    (1, 1 << 30, 1, 128),               # rows of a key-value head: a multiple of 2^32
    (1, 1 << 25, 1, 64),                # 2^31
    (1, 8200, 1, 1), (1, 16384, 128, 65),
    (1 << 30, 1 << 30, 1 << 30, 16), (70000, 1, 1, 1), (1024, 128, 128, 61),
])
def test_attention_workspaces_of_refused_sizes(L, B, H, Hkv, nq_max):
    """More rows or pairs than a call may have: 0 as for the other refusals, whatever the sizes multiply to."""
    from paper_2512_21857_amd import abi
    assert L.adt_tree_attn_weights_workspace_size(B, H, Hkv, 64, nq_max, 4096, abi.BF16) == 0
    assert L.adt_sparse_tree_attn_workspace_size(B, H, Hkv, 64, nq_max, 4096, 64, 16, abi.BF16) == 0


def test_attention_workspaces_at_the_limits(L):
    from paper_2512_21857_amd import abi
    for dtype in (abi.BF16, abi.F32):
        for B, H, Hkv, nq in ((1, 8192, 1, 1), (1, 64, 1, 128), (65535, 1, 1, 128), (1, 65535, 65535, 1)):
            assert L.adt_tree_attn_weights_workspace_size(B, H, Hkv, 64, nq, 100, dtype) > 0
            assert L.adt_sparse_tree_attn_workspace_size(B, H, Hkv, 64, nq, 100, 32, 3, dtype) > 0
    assert L.adt_sparse_tree_attn_workspace_size(1, 8, 8, 64, 1, 32 * 16384, 32, 8, abi.BF16) > 0
    assert L.adt_sparse_tree_attn_workspace_size(1, 8, 8, 64, 1, 32 * 16384 + 1, 32, 8, abi.BF16) == 0


EVICT = dict(k=FAKE, v=FAKE, w=FAKE, sb=2 * 64 * 100, ss=64 * 100, wb=200, ws=100, kv_len=FAKE, B=2, slices=2, Dh=64, cap=100,
             budget=40, n_first=4, n_last=8, ko=2 * FAKE, vo=2 * FAKE, wo=2 * FAKE, osb=2 * 64 * 40, oss=64 * 40, owb=80, ows=40,
             kept=FAKE, new_len=FAKE, dtype=1, stream=None)


@pytest.mark.parametrize("changed,code", [
    (dict(k=None), "E_ARG"), (dict(w=None), "E_ARG"), (dict(wo=None), "E_ARG"), (dict(kept=None), "E_ARG"),
    (dict(new_len=None), "E_ARG"), (dict(dtype=2), "E_ARG"), (dict(slices=0), "E_ARG"), (dict(budget=0), "E_ARG"),
    (dict(n_first=-1), "E_ARG"), (dict(n_first=20, n_last=21), "E_ARG"), (dict(Dh=65), "E_SHAPE"),
    (dict(Dh=8200, sb=1 << 30, ss=1 << 22, osb=1 << 30, oss=1 << 22), "E_SHAPE"), (dict(ko=FAKE), "E_ARG"),
    (dict(ko=FAKE, vo=FAKE, wo=FAKE), "E_SHAPE"), (dict(ss=64 * 99), "E_SHAPE"), (dict(ws=99), "E_SHAPE"),
    (dict(oss=64 * 39), "E_SHAPE"), (dict(ows=39), "E_SHAPE"), (dict(osb=64 * 40), "E_SHAPE"), (dict(wb=100), "E_SHAPE"),
    (dict(k=FAKE + 8), "E_SHAPE"), (dict(ss=64 * 100 + 4, sb=4 * 64 * 100), "E_SHAPE"),
])
def test_kv_evict_refusals(L, changed, code):
    from paper_2512_21857_amd import abi
    assert call(L.adt_kv_evict, EVICT, **changed) == getattr(abi, code), changed
    assert "kv_evict" in abi.last_error()


WCOMPACT = dict(w=FAKE, B=2, slices=2, wb=200, ws=100, kv_len=FAKE, cap=100, path=FAKE, path_stride=5, n_acc=FAKE, a_max=4,
                stream=None)


@pytest.mark.parametrize("changed,code", [
    (dict(w=None), "E_ARG"), (dict(path=None), "E_ARG"), (dict(B=0), "E_ARG"), (dict(a_max=128, path_stride=200), "E_CAPACITY"),
    (dict(a_max=5), "E_CAPACITY"), (dict(ws=99), "E_SHAPE"), (dict(wb=100), "E_SHAPE"),
])
def test_weights_compact_refusals(L, changed, code):
    from paper_2512_21857_amd import abi
    assert call(L.adt_weights_compact, WCOMPACT, **changed) == getattr(abi, code), changed
    assert call(L.adt_weights_compact, WCOMPACT, a_max=0) == abi.OK


@pytest.mark.parametrize("cap", [(1 << 31) - 1, (1 << 31) - (1 << 24) + 1])
def test_capacities_near_the_end_of_32_bits(L, cap):
    """Slots are indexed in 32 bits, up to a round past the last one: capacities that leave no room for it
    are refused, not read at negative slots."""
    from paper_2512_21857_amd import abi
    far = 1 << 45
    assert call(L.adt_kv_evict, EVICT, B=1, cap=cap, sb=far, ss=far, wb=far, ws=far) == abi.E_CAPACITY
    assert "kv_cap" in abi.last_error()
    assert call(L.adt_block_keys, KEYS, B=1, cap=cap, sb=far, sh=far, mb=far, mh=far) == abi.E_CAPACITY
    assert "kv_cap" in abi.last_error()
    assert call(L.adt_tree_attn_weights, RATED, B=1, cap=cap, sb=far, sh=far, wb=far, wh=far, ws_bytes=far) == abi.E_CAPACITY
    assert "kv_cap" in abi.last_error()
    assert L.adt_tree_attn_weights_workspace_size(1, 4, 2, 64, 8, cap, abi.BF16) == 0
    assert L.adt_tree_attn_weights_workspace_size(1, 4, 2, 64, 8, (1 << 31) - (1 << 24), abi.BF16) > 0


def test_runtime_needs_no_private_names_of_torch():
    """The wrappers import, and ask the public calls, where torch has no raw device and stream queries."""
    code = """
import torch
for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
from types import SimpleNamespace
torch.cuda.current_device = lambda: 3
torch.cuda.current_stream = lambda dev=None: SimpleNamespace(cuda_stream=100 + dev)
from paper_2512_21857_amd import runtime
seen = []
runtime._on_device(3, lambda *a: seen.append(a) or 0, (1, 2))
assert seen == [(1, 2, 103)], seen
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr


def test_more_slices_than_a_launch(L):
    """Slices whose launches would wrap at 2^32 threads are refused, not left out in silence."""
    from paper_2512_21857_amd import abi
    far = 1 << 45
    wide = dict(B=1, sb=far, wb=far, osb=far, owb=far)
    place = dict(ko=FAKE, vo=FAKE, wo=FAKE, oss=EVICT["ss"], ows=EVICT["ws"])
    assert call(L.adt_kv_evict, EVICT, slices=1 << 24, **wide) == abi.E_SHAPE
    assert "slices" in abi.last_error()
    assert call(L.adt_kv_evict, EVICT, slices=1 << 23, **wide, **place) == abi.E_SHAPE
    assert "slices" in abi.last_error()
    assert call(L.adt_weights_compact, WCOMPACT, B=1, slices=1 << 25, wb=far) == abi.E_SHAPE
    assert "slices" in abi.last_error()


def test_one_destination_for_keys_and_values(L):
    """Keys and values moved within one cache, each from where the other wrote, would lose rows."""
    from paper_2512_21857_amd import abi
    place = dict(wo=FAKE, osb=EVICT["sb"], oss=EVICT["ss"], owb=EVICT["wb"], ows=EVICT["ws"])
    assert call(L.adt_kv_evict, EVICT, ko=FAKE, vo=FAKE, **place) == abi.E_ARG                  # one cache, in place
    assert "destination" in abi.last_error()
    assert call(L.adt_kv_evict, EVICT, v=3 * FAKE, ko=2 * FAKE, vo=2 * FAKE) == abi.E_ARG       # two into one
    assert "destination" in abi.last_error()


def test_strides_of_dimensions_of_one():
    """A dimension of one has whatever stride its view left there: caches that differ in nothing else go
    together, and those that differ in a stride that counts do not."""
    import torch
    from paper_2512_21857_amd import runtime as rt
    f = torch.float32
    layer = torch.zeros(1, 3, 2, 10, 64)[:, 1]                  # one sequence's layer of a larger cache
    own = torch.zeros(1, 2, 10, 64)
    assert layer.stride() != own.stride()
    for k, v in ((layer, own), (own, layer)):
        assert rt._caches(k, v, -1, f) == ((1, 2, 10, 64), 2 * 10 * 64, 10 * 64)
    one = torch.zeros(2, 3, 64).as_strided((2, 3, 1, 64), (192, 64, 7, 1))      # one slot
    assert rt._caches(one, torch.zeros(2, 3, 1, 64), -1, f) == ((2, 3, 1, 64), 192, 64)
    head = torch.zeros(2, 5, 10, 64)[:, 2:3]                    # one head of several: the sequences lie apart
    assert rt._caches(head, head, -1, f) == ((2, 1, 10, 64), 5 * 640, 640)
    assert rt._weights("w", torch.zeros(2, 3).as_strided((2, 3, 1), (3, 1, 9)), -1, 2, 3, 1) == (3, 1)
    for k, v in ((head, torch.zeros(2, 1, 10, 64)), (own, torch.zeros(1, 2, 10, 65)[..., :64]),
                 (own, torch.zeros(1, 2, 64, 10).transpose(2, 3)), (own, torch.zeros(1, 2, 20, 64)[:, :, ::2]),
                 (torch.zeros(1, 2, 10, 65)[..., :64],) * 2, (own, own.double())):
        with pytest.raises(ValueError):
            rt._caches(k, v, -1, f)
    with pytest.raises(ValueError):
        rt._weights("w", torch.zeros(2, 3, 8)[:, :, ::2], -1, 2, 3, 4)
