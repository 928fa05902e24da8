"""The paged cache without a GPU: the oracle's 8-bit rows against torch's conversion, and what the entry points refuse."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import serving_oracle as srv
from oracle import tsa_oracle as orc
from paper_2602_03216_amd import binding as tsa

FAKE, ODD, ODD4 = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008), ctypes.c_void_p(0x1002)


def test_oracle_codes_match_torch():
    bits = np.arange(1 << 16, dtype=np.uint32).astype(np.uint16)
    x = orc.bf16_to_f64(bits)
    bits = bits[np.isfinite(x) & (np.abs(x) <= 448)]
    t = torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(srv.e4m3_code(orc.bf16_to_f64(bits)), t)
    assert np.array_equal(srv.e4m3_value(t), torch.from_numpy(t).view(torch.float8_e4m3fn).double().numpy())


def test_oracle_rows_use_the_smallest_power():
    r = np.random.Generator(np.random.PCG64(5))
    bits = orc.f64_to_bf16(r.standard_normal((500, 64)) * 2.0 ** r.integers(-60, 60, (500, 1)))
    bits[3] = 0
    bits[4, 1:] = 0
    bits[4, 0] = orc.f64_to_bf16(np.array([448.0 * 2.0 ** 5]))[0]
    code, byte = srv.quantise_rows(bits)
    x, s = np.abs(orc.bf16_to_f64(bits)).max(-1), 2.0 ** (byte.astype(float) - 127)
    live = x > 0
    assert (x[live] <= 448 * s[live]).all() and (x[live] > 224 * s[live]).all() and byte[3] == 127 and byte[4] == 132
    # a value that does not underflow is off by half a step of its code at most
    back = srv.e4m3_value(code) * s[:, None]
    err, v = np.abs(back - orc.bf16_to_f64(bits)), np.abs(orc.bf16_to_f64(bits))
    assert (err <= np.maximum(2.0 ** -4 * v, 2.0 ** -10 * s[:, None])).all()


def _desc(**kw):
    a = dict(n_seqs=3, n_tokens=7, Hq=4, Hkv=2, d=64, page_size=16, n_pages=10, max_pages=4)
    a.update(kw)
    return tsa.make_cache_desc(**a)


def _write(desc, K=FAKE, V=FAKE, cu=FAKE, kv=FAKE, tab=FAKE, kp=FAKE, vp=FAKE, ks=None, vs=None):
    return tsa.load_library().tsa_cache_write(ctypes.byref(desc) if desc is not None else None, K, V, cu, kv, tab, kp, vp, ks, vs, None)


def _read(desc, kp=FAKE, vp=FAKE, ks=None, vs=None, kv=FAKE, tab=FAKE, L=8, K=FAKE, V=FAKE):
    return tsa.load_library().tsa_cache_read(ctypes.byref(desc) if desc is not None else None, kp, vp, ks, vs, kv, tab, L, K, V, None)


BAD_DESCS = [(dict(n_seqs=0), 1), (dict(n_seqs=(1 << 20) + 1), 2), (dict(n_tokens=-1), 1), (dict(n_tokens=1 << 27), 2), (dict(max_q=-1), 1), (dict(Hq=3), 1),
             (dict(Hkv=0), 1), (dict(Hq=2048), 2), (dict(d=96), 2), (dict(page_size=8), 2), (dict(page_size=48), 2), (dict(page_size=512), 2),
             (dict(n_pages=0), 1), (dict(max_pages=0), 1), (dict(max_pages=1 << 26), 2), (dict(format=2), 1), (dict(format=-1), 1), (dict(window=-1), 1),
             (dict(scale=-1.0), 1), (dict(scale=math.inf), 1), (dict(q_strides=(32, 64)), 1), (dict(k_strides=(128, 0)), 1), (dict(v_strides=(128, 60)), 1),
             (dict(v_strides=(128, 32)), 1), (dict(o_strides=(-256, 64)), 1), (dict(o_strides=(1 << 31, 64)), 2)]


@pytest.mark.parametrize("kw,rc", BAD_DESCS)
def test_bad_descriptors(kw, rc):
    assert _write(_desc(**kw)) == rc and _read(_desc(**kw)) == rc


def test_refused():
    arg = tsa.TSA_ERR_ARG
    assert _write(None) == arg and _read(None) == arg
    d, e = _desc(), _desc(format=tsa.TSA_CACHE_E4M3)
    for name in ("K", "V", "cu", "kv", "tab", "kp", "vp"):
        assert _write(d, **{name: None}) == arg, name
        assert _write(d, **{name: ODD4}) == arg, name
        if name not in ("cu", "kv", "tab"):
            assert _write(d, **{name: ODD}) == arg, name
        if name != "cu":
            assert _read(d, **{name: None}) == arg and _read(d, **{name: ODD4}) == arg, name
    assert _write(e) == arg and _read(e) == arg                                   # 8 bits without scales
    assert _write(e, ks=FAKE) == arg and _read(e, vs=FAKE) == arg
    assert _write(d, ks=FAKE, vs=FAKE) == arg and _read(d, ks=FAKE) == arg        # bf16 with them
    assert _read(d, L=-1) == arg and _read(d, L=1 << 30) == arg
    assert _read(_desc(n_seqs=1 << 20, Hq=1024, Hkv=1024), L=1000) == tsa.TSA_ERR_UNSUPPORTED
    assert _write(_desc(n_tokens=0), K=None, V=None) == tsa.TSA_OK and _read(d, L=0, K=None, V=None) == tsa.TSA_OK
    d = _desc(n_tokens=2, n_seqs=1)
    with pytest.raises(tsa.TsaError):
        tsa.tsa_cache_write(d, torch.zeros(2, 2, 64, dtype=torch.bfloat16), None, None, None, None, None, None)      # not on a GPU


def _attend(desc, Q=FAKE, kp=FAKE, vp=FAKE, ks=None, vs=None, cu=FAKE, kv=FAKE, tab=FAKE, O=FAKE, lse=None, ws=FAKE, n=1 << 40):
    return tsa.load_library().tsa_attend_cache(ctypes.byref(desc) if desc is not None else None, Q, kp, vp, ks, vs, cu, kv, tab, O, lse, ws, n, None)


@pytest.mark.parametrize("kw,rc", BAD_DESCS)
def test_attend_bad_descriptors(kw, rc):
    assert _attend(_desc(**kw)) == rc
    assert tsa.load_library().tsa_attend_cache_workspace_bytes(ctypes.byref(_desc(**kw))) == 0


def test_attend_refused():
    arg, small = tsa.TSA_ERR_ARG, tsa.TSA_ERR_WORKSPACE
    assert _attend(None) == arg
    d, e = _desc(), _desc(format=tsa.TSA_CACHE_E4M3)
    for name in ("Q", "kp", "vp", "cu", "kv", "tab", "O"):
        assert _attend(d, **{name: None}) == arg and _attend(d, **{name: ODD4}) == arg, name
    assert _attend(d, lse=ODD4) == arg and _attend(e) == arg and _attend(e, ks=FAKE) == arg and _attend(d, vs=FAKE) == arg
    need = tsa.load_library().tsa_attend_cache_workspace_bytes(ctypes.byref(d))
    assert need > 0 and _attend(d, n=need - 1) == small and _attend(d, ws=None) == small and _attend(d, ws=ctypes.c_void_p(0x1080)) == small
    assert _attend(_desc(n_tokens=1 << 22, Hq=1024, Hkv=1)) == tsa.TSA_ERR_UNSUPPORTED
    assert _attend(_desc(n_tokens=0), Q=None, O=None, ws=None, n=0) == tsa.TSA_OK
    assert _attend(d) == arg and "O is Q" in tsa.tsa_last_error()
    with pytest.raises(tsa.TsaError):
        tsa.alloc_attend_cache_workspace(_desc(d=80))
