"""Calls of more workgroups than one axis of a launch holds (2^24 of 256 threads)."""
import numpy as np
import pytest
import torch

from tests import gpu_util as gu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tsa():
    from paper_2602_03216_amd import binding
    binding.load_library(build_if_missing=False)
    return binding


@pytest.fixture(autouse=True)
def memory_back():
    yield
    torch.cuda.empty_cache()


def _ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=gu.DEV)


def test_rotary_of_many_rows(tsa):
    """16 rows a workgroup at one head: 34 GB, in place."""
    L, d = (1 << 28) + 40, 64
    freq, _ = tsa.tsa_rotary_frequencies(tsa.TSA_ROTARY_PLAIN, d, 10000.0)
    x = torch.ones(1, 1, L, d, dtype=torch.bfloat16, device=gu.DEV)
    tsa.tsa_rotary(tsa.make_rotary_desc(1, 1, 1, L, d, freq), x, None, x, None)
    step = 1 << 23
    for first in (0, (1 << 27) - step, 1 << 27, (1 << 28) - step, (1 << 28) - 60):
        n = min(step, L - first)
        y = torch.ones(1, 1, n, d, dtype=torch.bfloat16, device=gu.DEV)
        tsa.tsa_rotary(tsa.make_rotary_desc(1, 1, 1, n, d, freq, start=first), y, None, y, None)
        assert torch.equal(x[:, :, first:first + n], y), first


def test_read_of_many_rows(tsa):
    """32 rows a workgroup: 2^29 and more rows, 69 GB, which K and V share here (the pools are the same)."""
    n, H, page, d = 8, 4, 256, 64
    L = (1 << 24) + page
    pool = gu.to_dev(gu.rand_bits(np.random.Generator(np.random.PCG64(9000)), (3, H, page, d)))
    table = (torch.arange(L // page, dtype=torch.int32, device=gu.DEV)[None] + torch.arange(n, dtype=torch.int32, device=gu.DEV)[:, None]) % 3
    kv = [L - i for i in range(n)]
    desc = tsa.make_cache_desc(n, 0, H, H, d, page, 3, L // page)
    out = torch.full((n, H, L, d), 5.0, dtype=torch.bfloat16, device=gu.DEV)
    tsa.tsa_cache_read(desc, pool, pool, _ints(kv), table.contiguous(), L, out, out)
    for i in range(n):
        got = out[i].view(H, L // page, page, d)
        for p0 in range(0, L // page, 1 << 14):
            ids = table[i, p0:p0 + (1 << 14)].long()
            want = pool[ids].transpose(0, 1).contiguous()
            if p0 + (1 << 14) >= L // page and i:
                want.view(H, -1, d)[:, -i:] = 0              # behind its end
            assert torch.equal(got[:, p0:p0 + (1 << 14)], want), (i, p0)
