"""The paged cache against the oracle, bit for bit: rows in bf16 and in 8 bits, ragged and empty sequences, odd places, pages that are
not there, rows behind the last sequence, and sequences read back."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as srv
from oracle import tsa_oracle as orc
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tsa():
    from paper_2602_03216_amd import binding
    binding.load_library(build_if_missing=False)
    return binding


def _ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=gu.DEV)


def _tables(r, kv, page, spare=2):
    """A table with the pages of every sequence anywhere in the pool, -1 behind them."""
    need = [-(-k // page) for k in kv]
    ids = r.permutation(sum(need) + spare)
    tab = np.full((len(kv), max(1, max(need) + 1)), -1, dtype=np.int64)
    at = 0
    for i, n in enumerate(need):
        tab[i, :n] = ids[at:at + n]
        at += n
    return tab, sum(need) + spare


def _rows(r, shape):
    """Rows of very different sizes, zeros and exact powers among them."""
    x = r.standard_normal(shape) * 2.0 ** r.integers(-12, 12, shape[:-1])[..., None]
    flat = x.reshape(-1, shape[-1])
    flat[::7, ::3] = 0.0
    if len(flat) > 3:
        flat[1] = 0.0
        flat[2] = 2.0 ** 8 * 1.75
        flat[3, 0] = 2.0 ** 9 * 1.7578125 * 2
    return orc.f64_to_bf16(x)


CASES = [  # new tokens, cached tokens, Hkv, d, page, rows behind the last sequence
    ([1], [1], 1, 64, 16, 0),
    ([1, 0, 1, 1], [5, 17, 16, 33], 8, 128, 16, 0),
    ([3, 17, 0, 1], [3, 100, 0, 64], 5, 128, 32, 5),
    ([40], [555], 2, 64, 64, 0),
    ([5, 700], [700, 700], 3, 128, 256, 1),
    ([1] * 70, list(range(1, 71)), 4, 64, 16, 2),
    ([31, 0, 0, 2300], [31, 9, 0, 2301], 7, 128, 128, 0),       # more than 2048 tokens: four per wavefront
    ([2049], [2049], 1, 64, 16, 3),
]


@pytest.mark.parametrize("e4m3", [0, 1])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_write_and_read(tsa, case, e4m3):
    new, kv, H, d, page, pad = CASES[case]
    r = np.random.Generator(np.random.PCG64(5000 + case))
    n, T = len(new), sum(new) + pad
    cu = np.concatenate([[0], np.cumsum(new)])
    tab, n_pages = _tables(r, kv, page)
    kw = {}
    row = _rows(r, (T, 3 * H, d))                          # K and V out of the rows of a projection
    dev = gu.to_dev(row)
    kw = dict(k_strides=(3 * H * d, d), v_strides=(3 * H * d, d))
    desc = tsa.make_cache_desc(n, T, H, H, d, page, n_pages, tab.shape[1], tsa.TSA_CACHE_E4M3 if e4m3 else tsa.TSA_CACHE_BF16, **kw)
    shape = (n_pages, H, page, d)
    pools = [torch.full(shape, 77, dtype=torch.uint8 if e4m3 else torch.int16, device=gu.DEV) for _ in "kv"]
    scales = [torch.full(shape[:3], 99, dtype=torch.uint8, device=gu.DEV) if e4m3 else None for _ in "kv"]
    typed = [p if e4m3 else p.view(torch.bfloat16) for p in pools]
    tsa.tsa_cache_write(desc, dev[:, H:2 * H], dev[:, 2 * H:], _ints(cu), _ints(kv), _ints(tab), *typed, *scales)
    for which, (pool, scale) in enumerate(zip(pools, scales)):
        src = row[:, (1 + which) * H:(2 + which) * H]
        want = np.full(shape, 77, dtype=np.uint8 if e4m3 else np.uint16)
        wants = np.full(shape[:3], 99, dtype=np.uint8)
        code, byte = srv.quantise_rows(src) if e4m3 else (src, None)
        for t, p, o in srv.places(cu, kv, tab, page, n_pages, T):
            want[p, :, o] = code[t]
            if e4m3:
                wants[p, :, o] = byte[t]
        got = pool.cpu().numpy() if e4m3 else pool.cpu().numpy().view(np.uint16)
        assert np.array_equal(got, want)
        if e4m3:
            assert np.array_equal(scale.cpu().numpy(), wants)
    # every sequence back, some positions beyond the longest one too
    L = max(kv) + 3
    K, V = (torch.full((n, H, L, d), 5.0, dtype=torch.bfloat16, device=gu.DEV) for _ in "kv")
    full = [np.random.Generator(np.random.PCG64(5100 + w)).integers(0, 256 if e4m3 else 1 << 16, shape).astype(np.uint8 if e4m3 else np.uint16) for w in (0, 1)]
    if e4m3:
        full = [np.where(f & 0x7f == 0x7f, 3, f).astype(np.uint8) for f in full]
        sc = [np.random.Generator(np.random.PCG64(5200 + w)).integers(100, 150, shape[:3]).astype(np.uint8) for w in (0, 1)]
    for w in (0, 1):
        pools[w].copy_(torch.from_numpy(full[w] if e4m3 else full[w].view(np.int16)))
        if e4m3:
            scales[w].copy_(torch.from_numpy(sc[w]))
    tsa.tsa_cache_read(desc, *typed, _ints(kv), _ints(tab), L, K, V, *scales)
    for w, out in ((0, K), (1, V)):
        want = np.zeros((n, H, L, d), dtype=np.uint16)
        for i in range(n):
            for p in range(kv[i]):
                rows = full[w][tab[i, p // page], :, p % page]
                want[i, :, p] = rows if not e4m3 else orc.f64_to_bf16(srv.e4m3_value(rows) * 2.0 ** (sc[w][tab[i, p // page], :, p % page].astype(float) - 127)[:, None])
        assert np.array_equal(gu.from_dev(out), want)


def test_every_finite_value_in_eight_bits(tsa):
    """Every bf16 value beside a largest one of its own size, and beside ones 2^1 to 2^9 times as large: rounding, ties and the small end."""
    bits = np.arange(1 << 15, dtype=np.uint32).astype(np.uint16)
    x = orc.bf16_to_f64(bits)
    bits = bits[np.isfinite(x)]
    rows = []
    for k in range(10):
        body = np.resize(bits, (-(-len(bits) // 63), 63))
        top = np.abs(orc.bf16_to_f64(body)).max(-1)
        lead = orc.f64_to_bf16(np.minimum(top * 2.0 ** k, 3.0e38))
        rows.append(np.concatenate([lead[:, None], body | np.uint16(0x8000 if k % 2 else 0)], 1))
    rows = np.concatenate(rows)[:, None]                   # [T, 1, 64]
    T = len(rows)
    pages = -(-T // 256)
    desc = tsa.make_cache_desc(1, T, 1, 1, 64, 256, pages, pages, tsa.TSA_CACHE_E4M3)
    kp, vp = (torch.zeros(pages, 1, 256, 64, dtype=torch.uint8, device=gu.DEV) for _ in "kv")
    ks, vs = (torch.zeros(pages, 1, 256, dtype=torch.uint8, device=gu.DEV) for _ in "kv")
    dev = gu.to_dev(rows)
    tsa.tsa_cache_write(desc, dev, dev, _ints([0, T]), _ints([T]), _ints([range(pages)]), kp, vp, ks, vs)
    code, byte = srv.quantise_rows(rows)
    assert np.array_equal(kp.cpu().numpy().reshape(-1, 64)[:T], code[:, 0]) and np.array_equal(ks.cpu().numpy().reshape(-1)[:T], byte[:, 0])
    assert torch.equal(kp, vp) and torch.equal(ks, vs)


def test_pages_that_are_not_there_and_lengths_that_do_not_fit(tsa):
    """Ids outside the pool, more new tokens than cached ones, lengths beyond the table: nothing is touched but what is described."""
    r = np.random.Generator(np.random.PCG64(5300))
    H, d, page, n_pages = 2, 128, 16, 6
    new, kv = [20, 9, 2], [20, 4, 33]
    tab = np.array([[4, -1, 7], [1 << 30, 2, 0], [3, 0, 5]])
    tab[0, 1] = n_pages
    cu = np.concatenate([[0], np.cumsum(new)])
    T = sum(new)
    desc = tsa.make_cache_desc(3, T, H, H, d, page, n_pages, 3)
    src = gu.rand_bits(r, (T, H, d))
    kp, vp = (torch.full((n_pages, H, page, d), 3.0, dtype=torch.bfloat16, device=gu.DEV) for _ in "kv")
    tsa.tsa_cache_write(desc, gu.to_dev(src), gu.to_dev(src), _ints(cu), _ints(kv), _ints(tab), kp, vp)
    want = np.full((n_pages, H, page, d), orc.f64_to_bf16(np.array([3.0]))[0], dtype=np.uint16)
    where = srv.places(cu, kv, tab, page, n_pages, T)
    assert {p for _, p, _ in where} == {4, 0, 5}
    for t, p, o in where:
        want[p, :, o] = src[t]
    assert np.array_equal(gu.from_dev(kp), want) and torch.equal(kp, vp)
    K, V = (torch.full((3, H, 40, d), 5.0, dtype=torch.bfloat16, device=gu.DEV) for _ in "kv")
    tsa.tsa_cache_read(desc, kp, vp, _ints([40, 4, 1 << 30]), _ints(tab), 40, K, V)
    back = np.zeros((3, H, 40, d), dtype=np.uint16)
    for i, n in enumerate([40, 4, 40]):
        for p in range(n):
            if 0 <= tab[i, p // page] < n_pages:
                back[i, :, p] = want[tab[i, p // page], :, p % page]
    assert np.array_equal(gu.from_dev(K), back) and torch.equal(K, V)


def test_a_pool_beyond_four_gigabytes(tsa):
    """Rows whose place does not fit 32 bits."""
    H, d, page, n_pages = 8, 128, 256, 9000                # 4.7 GB per pool
    r = np.random.Generator(np.random.PCG64(5400))
    kp, vp = (torch.empty(n_pages, H, page, d, dtype=torch.bfloat16, device=gu.DEV) for _ in "kv")
    src = gu.rand_bits(r, (300, H, d))
    tab = [[8999, 5]]
    desc = tsa.make_cache_desc(1, 300, H, H, d, page, n_pages, 2)
    tsa.tsa_cache_write(desc, gu.to_dev(src), gu.to_dev(src), _ints([0, 300]), _ints([300]), _ints(tab), kp, vp)
    assert np.array_equal(gu.from_dev(kp[8999]), src[:256].transpose(1, 0, 2)) and np.array_equal(gu.from_dev(vp[5, :, :44]), src[256:].transpose(1, 0, 2))
    K, V = (torch.zeros(1, H, 300, d, dtype=torch.bfloat16, device=gu.DEV) for _ in "kv")
    tsa.tsa_cache_read(desc, kp, vp, _ints([300]), _ints(tab), 300, K, V)
    assert np.array_equal(gu.from_dev(K)[0], src.transpose(1, 0, 2)) and torch.equal(K, V)


def test_captured(tsa):
    H, d, page = 4, 128, 16
    r = np.random.Generator(np.random.PCG64(5500))
    desc = tsa.make_cache_desc(2, 6, H, H, d, page, 8, 4, tsa.TSA_CACHE_E4M3)
    x = torch.empty(6, H, d, dtype=torch.bfloat16, device=gu.DEV)
    kp, vp = (torch.zeros(8, H, page, d, dtype=torch.uint8, device=gu.DEV) for _ in "kv")
    ks, vs = (torch.zeros(8, H, page, dtype=torch.uint8, device=gu.DEV) for _ in "kv")
    cu, kv, tab = _ints([0, 2, 6]), _ints([2, 4]), _ints([[0, 1, 2, 3], [4, 5, 6, 7]])
    K, V = (torch.zeros(2, H, 64, d, dtype=torch.bfloat16, device=gu.DEV) for _ in "kv")

    def step():
        tsa.tsa_cache_write(desc, x, x, cu, kv, tab, kp, vp, ks, vs)
        tsa.tsa_cache_read(desc, kp, vp, kv, tab, 64, K, V, ks, vs)

    x.copy_(gu.to_dev(gu.rand_bits(r, (6, H, d))))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):                                    # the lengths grow from replay to replay
        x.copy_(gu.to_dev(gu.rand_bits(r, (6, H, d))))
        kv.copy_(_ints([2 + 15 * k, 4 + 18 * k]))
        graph.replay()
        torch.cuda.synchronize()
        got = K.clone(), V.clone(), kp.clone(), ks.clone()
        K.fill_(1.0)
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (K, V, kp, ks)))
        assert K[1, :, 4 + 18 * k:].abs().max() == 0 and K[1, :, :4 + 18 * k].abs().sum() > 0


def test_values_that_are_no_numbers(tsa):
    """8 bits: they become NaN, and the row's exponent is the largest; the rows beside them are as without them."""
    K = torch.randn(5, 2, 64, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).to(gu.DEV)
    bad = K.clone()
    bad[0, 0, 3], bad[1, 0, 4], bad[2, 1, 5] = float("inf"), float("nan"), -float("inf")
    desc = tsa.make_cache_desc(1, 5, 2, 2, 64, 16, 1, 1, tsa.TSA_CACHE_E4M3)
    pools = []
    for x in (K, bad):
        kp, ks = torch.zeros(1, 2, 16, 64, dtype=torch.uint8, device=gu.DEV), torch.zeros(1, 2, 16, dtype=torch.uint8, device=gu.DEV)
        tsa.tsa_cache_write(desc, x, x, _ints([0, 5]), _ints([5]), _ints([[0]]), kp, kp.clone(), ks, ks.clone())
        pools.append((kp[0].cpu(), ks[0].cpu()))
    (kp, ks), (kp2, ks2) = pools
    for t, h, i in ((0, 0, 3), (1, 0, 4), (2, 1, 5)):
        assert ks2[h, t] == 247 and kp2[h, t, i] & 0x7f == 0x7f and (kp2[h, t] & 0x7f == 0x7f).sum() == 1
        kp2[h, t], ks2[h, t] = kp[h, t], ks[h, t]
    assert torch.equal(kp, kp2) and torch.equal(ks, ks2)
