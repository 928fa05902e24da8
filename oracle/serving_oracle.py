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
