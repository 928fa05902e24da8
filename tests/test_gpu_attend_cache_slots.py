"""tsa_attend_cache where many sequences share a call with prompts, or the caller does not know that none has one: the slots of the row tiles
are then counted by rows instead of by sequences."""
import pytest

from tests.test_gpu_attend_cache import Batch, tsa  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu

CASES = {
    # one head a group: rows are tokens, and 65 is the fewest that go by rows; 64.5 of them are a slot
    "tight": dict(new=[65, 65, 1, 129, 64, 65, 0, 257, 2, 65, 193, 0, 65] + [1] * 8, Hq=2, Hkv=2, d=64, page=16),
    "tight_window": dict(new=[1, 65, 65, 65, 130, 66, 129, 64] + [1] * 9, Hq=1, Hkv=1, d=128, page=32, window=300),
    "prompts_among_single_tokens": dict(new=[1] * 90 + [150] + [1] * 60 + [17, 33, 1, 1, 0, 20], Hq=8, Hkv=2, d=128, page=16, pad=3),
    "last": dict(new=[1] * 66 + [300], Hq=4, Hkv=1, d=64, page=64),
    "first": dict(new=[300] + [1] * 66, Hq=4, Hkv=1, d=128, page=64, pad=1),
    "single_tokens_only": dict(new=[1] * 64, Hq=8, Hkv=2, d=128, page=16),
}


@pytest.mark.parametrize("e4m3", [0, 1])
@pytest.mark.parametrize("name", list(CASES))
def test_slots_by_rows(tsa, name, e4m3):  # noqa: F811
    c = CASES[name]
    # contexts of many parts for the prompts, short ones beside them
    kv = [x + (1700 + 40 * i) * (x > 16) + 37 * i % 500 for i, x in enumerate(c["new"])]
    b = Batch(8000 + list(CASES).index(name), kv=kv, e4m3=e4m3, **c)
    rows, g = b.T * b.Hq // b.Hkv, b.Hq // b.Hkv
    assert 2 * rows // 129 < rows // 128 + len(kv) and (name == "single_tokens_only" or max(c["new"]) * g > 64)      # (the case is what it says)
    for max_q in (0, max(c["new"])):
        b.check(*b.run(tsa, max_q=max_q))
