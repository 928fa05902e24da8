"""Rotary positions without a GPU: the frequencies against their closed forms, and what the entry points refuse."""
import ctypes
import math

import pytest

from paper_2602_03216_amd import binding as tsa

FAKE = ctypes.c_void_p(0x1000)        # aligned, never dereferenced: validation fails first


def test_plain_linear_and_raised_base():
    for rot, base in ((128, 10000.0), (32, 500000.0), (2, 10.0)):
        want = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
        freq, gain = tsa.tsa_rotary_frequencies(tsa.TSA_ROTARY_PLAIN, rot, base)
        assert gain == 1.0 and freq == pytest.approx(want, rel=1e-14)
        freq, gain = tsa.tsa_rotary_frequencies(tsa.TSA_ROTARY_LINEAR, rot, base, 4.0)
        assert gain == 1.0 and freq == pytest.approx([f / 4 for f in want], rel=1e-14)
    # the raised base leaves the first pair alone and stretches the last one by the factor
    freq, gain = tsa.tsa_rotary_frequencies(tsa.TSA_ROTARY_BASE, 64, 10000.0, 8.0)
    assert freq[0] == 1.0 and freq[31] == pytest.approx(10000.0 ** (-62 / 64) / 8, rel=1e-13)


def test_stretched_by_parts():
    rot, base, factor, orig = 128, 10000.0, 8.0, 32768.0
    plain = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    freq, gain = tsa.tsa_rotary_frequencies(tsa.TSA_ROTARY_PARTS, rot, base, factor, orig)
    assert gain == pytest.approx(0.1 * math.log(8.0) + 1, rel=1e-7)
    turns = [orig * f / (2 * math.pi) for f in plain]
    lo = max(i for i in range(64) if turns[i] > 32)                # the ramp starts at or just above this pair ...
    hi = min(i for i in range(64) if turns[i] < 1)                 # ... and ends at this one
    for i, (f, p) in enumerate(zip(freq, plain)):
        share = min(1.0, max(0.0, (i - lo) / (hi - lo)))
        assert f == pytest.approx(p * (1 - share) + p / factor * share, rel=1e-12), i


def test_stretched_by_wavelength():
    rot, base, factor, orig = 64, 500000.0, 4.0, 8192.0
    freq, gain = tsa.tsa_rotary_frequencies(tsa.TSA_ROTARY_WAVELENGTH, rot, base, factor, orig, 4.0, 1.0)
    assert gain == 1.0
    kinds = set()
    for i, f in enumerate(freq):
        p = base ** (-2.0 * i / rot)
        turns = orig * p / (2 * math.pi)
        if turns >= 4:
            want, kind = p, "kept"
        elif turns <= 1:
            want, kind = p / factor, "stretched"
        else:
            s = (turns - 1) / 3
            want, kind = s * p + (1 - s) * p / factor, "between"
        kinds.add(kind)
        assert f == pytest.approx(want, rel=1e-12), i
    assert kinds == {"kept", "stretched", "between"}


@pytest.mark.parametrize("args", [(5, 64, 1e4, 2.0, 4096.0), (-1, 64, 1e4), (0, 63, 1e4), (0, 0, 1e4), (0, 130, 1e4), (0, 64, 1.0), (0, 64, math.inf),
                                  (1, 64, 1e4, 0.5), (1, 64, 1e4, math.nan), (2, 2, 1e4, 2.0), (3, 64, 1e4, 2.0, 0.0), (3, 64, 1e4, 2.0, 4096.0, 1.0, 2.0),
                                  (4, 64, 1e4, 2.0, 4096.0, 4.0, -1.0)])
def test_frequencies_refused(args):
    with pytest.raises(tsa.TsaError) as e:
        tsa.tsa_rotary_frequencies(*args)
    assert e.value.code == tsa.TSA_ERR_ARG


def _call(desc, Q=FAKE, K=FAKE, pos=FAKE, Qo=FAKE, Ko=FAKE):
    return tsa.load_library().tsa_rotary(ctypes.byref(desc) if desc is not None else None, Q, K, pos, Qo, Ko, None)


def _desc(rot=64, **kw):
    a = dict(B=2, Hq=4, Hkv=2, L=10, d=64)
    a.update({k: kw.pop(k) for k in list(kw) if k in a})
    return tsa.make_rotary_desc(**a, freq=[1.0] * (rot // 2), **kw)


def test_rotary_refused():
    arg, uns = tsa.TSA_ERR_ARG, tsa.TSA_ERR_UNSUPPORTED
    assert _call(None) == arg
    for kw, rc in ((dict(B=0), arg), (dict(L=-1), arg), (dict(Hq=0), arg), (dict(Hkv=-3), arg), (dict(Hq=70000), arg), (dict(d=96), uns), (dict(rot=24), uns),
                   (dict(rot=0), uns), (dict(rot=128), uns), (dict(rot=128, d=64), uns), (dict(interleaved=2), arg), (dict(gain=math.nan), arg),
                   (dict(q_strides=(0, 64, 60)), arg), (dict(q_strides=(640, 4, 64)), arg), (dict(q_strides=(0, 640, 64)), arg),
                   (dict(k_strides=(1280, 0, 64)), arg), (dict(k_out_strides=(-1280, 640, 64)), arg), (dict(q_out_strides=(1 << 50, 640, 64)), uns),
                   (dict(B=1 << 16, L=1 << 16), uns)):
        assert _call(_desc(**kw)) == rc, kw
    odd = ctypes.c_void_p(0x1008)
    d = _desc()
    assert _call(d, Q=odd) == arg and _call(d, Ko=odd) == arg and _call(d, pos=ctypes.c_void_p(0x1002)) == arg
    assert _call(d, Q=None) == arg and _call(d, Ko=None) == arg and _call(d, None, None, FAKE, None, None) == arg
    assert _call(_desc(start=(1 << 31) - 5), pos=None) == arg
    # an output that is its input has to lie as the input does
    assert _call(_desc(q_out_strides=(2560, 64, 256))) == arg and "strides" in tsa.tsa_last_error()
    bad = _desc()
    bad.freq[3] = math.inf
    assert _call(bad) == arg
    bad = _desc()
    bad.reserved = 1
    assert _call(bad) == arg
    assert _call(_desc(L=0)) == tsa.TSA_OK                  # nothing to do


def test_binding_checks_tensors():
    import torch
    d = _desc(B=1, L=3)
    x = torch.zeros(1, 4, 3, 64, dtype=torch.bfloat16)
    with pytest.raises(tsa.TsaError):
        tsa.tsa_rotary(d, x, None, x, None)                  # not on a GPU
    with pytest.raises(tsa.TsaError):
        tsa.make_rotary_desc(1, 4, 4, 3, 128, [1.0] * 65)
