"""CPU oracle of the operators that stand beside the prefill layer (rotary positions, the paged cache, attention over it): float64
numpy, one definition after the other, no blocking and no fusion.  bf16 tensors come as their bit patterns (uint16)."""
import numpy as np

from oracle.tsa_oracle import bf16_to_f64


def rotary(x_bits, positions, freq, gain=1.0, interleaved=False):
    """x_bits [B,H,L,d], positions [B,L] -> float64 [B,H,L,d]."""
    x = bf16_to_f64(x_bits)
    out = x.copy()
    rot = 2 * len(freq)
    a = np.asarray(positions, dtype=np.float64)[:, None, :, None] * np.asarray(freq, dtype=np.float64)
    first = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
    second = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
    out[..., first] = gain * (x[..., first] * np.cos(a) - x[..., second] * np.sin(a))
    out[..., second] = gain * (x[..., first] * np.sin(a) + x[..., second] * np.cos(a))
    return out


E4M3_VALUES = np.array([m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


def e4m3_code(x):
    """Code of the nearest value of the format (of two as near, the one with the even code); |x| <= 448."""
    x = np.asarray(x, dtype=np.float64)
    y = np.abs(x)
    hi = np.clip(np.searchsorted(E4M3_VALUES, y), 1, 126)
    lo = hi - 1
    down, up = y - E4M3_VALUES[lo], E4M3_VALUES[hi] - y
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def e4m3_value(code):
    code = np.asarray(code, dtype=np.int64)
    return np.where(code & 128, -1.0, 1.0) * E4M3_VALUES[code & 127]


def quantise_rows(x_bits):
    """Rows of bf16 as (codes, bytes): x = e4m3(code) * 2^(byte - 127) up to the rounding of the code."""
    x = bf16_to_f64(x_bits)
    big = np.abs(x).max(-1)
    e = np.full(big.shape, -126, dtype=np.int64)
    for k in range(-126, 128):                            # the smallest e with big <= 448 * 2^e
        e = np.where((big > 448.0 * 2.0 ** (k - 1)) & (k > -126), k, e)
    e = np.where(big == 0, 0, e)
    return e4m3_code(x / 2.0 ** e[..., None].astype(np.float64)), (e + 127).astype(np.uint8)


def places(cu_q, kv_len, table, page_size, n_pages, n_tokens):
    """(token, page, row of the page) of every new token that is written."""
    out = []
    for i in range(len(kv_len)):
        for t in range(cu_q[i], min(cu_q[i + 1], n_tokens)):
            p = kv_len[i] - (cu_q[i + 1] - t)
            if p >= 0 and 0 <= table[i][p // page_size] < n_pages:
                out.append((t, table[i][p // page_size], p % page_size))
    return out


def attend(q, k, v, there, scale, window=0):
    """q [n,d] at the last n positions of k, v [L,d] (float64); there [L]: whether a key's page is -> out [n,d], lse [n], and the same
    average of |v| (what an error of the probabilities is measured by)."""
    n, L = len(q), len(k)
    p, t = np.arange(L - n, L)[:, None], np.arange(L)[None, :]
    seen = (t <= p) & there[None, :]
    if window:
        seen &= t > p - window
    s = np.where(seen, (q @ np.where(there[:, None], k, 0.0).T) * scale, -np.inf)
    m = s.max(-1, keepdims=True, initial=-1e300)
    w = np.exp(s - m)
    l = w.sum(-1, keepdims=True)
    v = np.where(there[:, None], v, 0.0)
    with np.errstate(divide="ignore", invalid="ignore"):
        mean = lambda x: np.where(l > 0, (w @ x) / l, 0.0)
        return mean(v), np.where(l > 0, m + np.log(l), -np.inf)[:, 0], mean(np.abs(v))
