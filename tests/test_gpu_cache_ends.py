"""8-bit rows with every exponent there is, read back: what bf16 cannot hold is rounded as bf16 is, to nearest even, down to nothing and up to infinity."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as srv
from oracle import tsa_oracle as orc
from tests import gpu_util as gu
from tests.test_gpu_cache import tsa  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def test_every_code_under_every_exponent(tsa):  # noqa: F811
    codes = np.array([c for c in range(256) if c & 0x7f != 0x7f], dtype=np.uint8)
    rows = np.resize(codes, (4, 64))                       # 254 codes in four rows of a page of 1024 rows: exponents 1 .. 254 of each
    pool, scales = np.repeat(rows, 254, 0), np.tile(np.arange(1, 255, dtype=np.uint8), 4)
    L, page = 4 * 254, 256
    full = np.zeros((4 * page, 64), dtype=np.uint8)
    sc = np.full(4 * page, 127, dtype=np.uint8)
    full[:L], sc[:L] = pool, scales
    kp = torch.from_numpy(full.reshape(4, 1, page, 64)).to(gu.DEV)
    ks = torch.from_numpy(sc.reshape(4, 1, page)).to(gu.DEV)
    desc = tsa.make_cache_desc(1, 0, 1, 1, 64, page, 4, 4, tsa.TSA_CACHE_E4M3)
    K, V = (torch.full((1, 1, L, 64), 5.0, dtype=torch.bfloat16, device=gu.DEV) for _ in "kv")
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=gu.DEV)
    tsa.tsa_cache_read(desc, kp, kp, ints([L]), ints([[0, 1, 2, 3]]), L, K, V, ks, ks)
    with np.errstate(over="ignore"):
        want = torch.from_numpy(srv.e4m3_value(pool) * 2.0 ** (scales.astype(float) - 127)[:, None]).to(torch.float32).to(torch.bfloat16)
    got = K[0, 0].cpu()
    bad = (got.view(torch.int16) != want.view(torch.int16)).nonzero()
    assert len(bad) == 0, (len(bad), [(scales[r], hex(pool[r, c]), got[r, c].item(), want[r, c].item()) for r, c in bad[:8].tolist()])
    assert torch.equal(K.view(torch.int16), V.view(torch.int16))
