"""tsa_attend_cache with softmax scales at the ends of what it takes: an average of all keys, and the row of V of the largest logit."""
import numpy as np
import pytest

from oracle import tsa_oracle as orc
from tests import gpu_util as gu
from tests.test_gpu_attend_cache import Batch, tsa  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [0, 1])
@pytest.mark.parametrize("new", [[1], [200]])
def test_a_scale_that_makes_all_keys_alike(tsa, new, e4m3):  # noqa: F811
    b = Batch(8500, new, [900], 4, 2, 128, 16, e4m3=e4m3, scale=2.0 ** -100)
    b.check(*b.run(tsa))


@pytest.mark.parametrize("e4m3", [0, 1])
@pytest.mark.parametrize("new,scale", [([1], 2.0 ** 20), ([200], 2.0 ** 20), ([1], 2.0 ** 24), ([200], 2.0 ** 24)])
def test_a_scale_that_leaves_one_key(tsa, new, scale, e4m3):  # noqa: F811
    """Logits of up to 2^29.  A logit is off by its 64 products' sum in 32 bits (64 * 2^-24 of the products' magnitudes, in whatever order) and by a step of what is kept
    of it and of the running maximum (2^-23 of the largest, each).  Where the largest leads by twice that and by 64 more the other keys have nothing, and its own
    probability is a power of two of that rounding, cut to bf16 (2^-8) but not in the sum it is divided by; 2^-8 more for the output."""
    b = Batch(8600, new, [900], 4, 2, 64, 16, e4m3=e4m3, scale=scale)
    O, lse = b.run(tsa)
    got, q, lse = orc.bf16_to_f64(gu.from_dev(O)), orc.bf16_to_f64(b.q), lse.double().cpu().numpy()
    assert np.isfinite(got).all() and np.isfinite(lse).all()
    K, V, _ = b.rows[0]
    for h in range(4):
        s, mag = (q[:, h] @ K[h // 2].T) * scale, (np.abs(q[:, h]) @ np.abs(K[h // 2]).T).max(-1) * scale
        s[np.arange(900)[None] > 900 - new[0] + np.arange(new[0])[:, None]] = -np.inf
        top = np.sort(s, -1)
        off = 64 * 2.0 ** -24 * mag + 2.0 ** -22 * np.abs(top[:, -1])
        clear = top[:, -1] - top[:, -2] > 2 * off + 64
        assert clear.mean() > 0.9
        want = V[h // 2][s.argmax(-1)]
        assert (np.abs(got[:, h] - want)[clear] <= (2.0 ** -8 + 2.0 ** -8 + 2.0 ** -15) * np.abs(want[clear])).all()
        assert (np.abs(lse[:, h] - top[:, -1]) <= off + 1)[clear].all()
