"""The operators of a long or bounded cache on the CPU: refusals, each before anything is
launched, and the host-only rotary frequencies against their formulas."""
import ctypes as C
import math

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
