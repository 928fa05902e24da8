"""The operators together, as a program uses them: prompts rotated, attended densely and by the sparse layer, their K and V kept in a paged cache,
then tokens one after another; what is computed from the cache against what the prefill entry points compute from whole tensors."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as srv
from oracle import tsa_oracle as orc
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu

Hq, Hkv, d, page = 8, 2, 128, 16


@pytest.fixture(scope="module")
def tsa():
    from paper_2602_03216_amd import binding
    binding.load_library(build_if_missing=False)
    return binding


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=gu.DEV)


def new(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype, device=gu.DEV)


class Cache:
    def __init__(self, tsa, n_seqs, max_len, e4m3, seed):
        self.tsa, self.n, self.e4m3 = tsa, n_seqs, e4m3
        self.max_pages = -(-max_len // page)
        self.n_pages = n_seqs * self.max_pages + 1
        ids = np.random.Generator(np.random.PCG64(seed)).permutation(self.n_pages)[:n_seqs * self.max_pages]
        self.table = ints(ids.reshape(n_seqs, self.max_pages))
        kind = torch.uint8 if e4m3 else torch.bfloat16
        self.pools = [new(self.n_pages, Hkv, page, d, dtype=kind) for _ in "kv"]
        self.scales = [new(self.n_pages, Hkv, page, dtype=torch.uint8) if e4m3 else None for _ in "kv"]

    def desc(self, n_tokens, **kw):
        return self.tsa.make_cache_desc(self.n, n_tokens, Hq, Hkv, d, page, self.n_pages, self.max_pages,
                                        self.tsa.TSA_CACHE_E4M3 if self.e4m3 else self.tsa.TSA_CACHE_BF16, **kw)


@pytest.mark.parametrize("e4m3", [0, 1])
def test_prompts_then_tokens(tsa, e4m3):
    r = np.random.Generator(np.random.PCG64(8000 + e4m3))
    lens, steps = [150, 333, 64], 3
    T = sum(lens)
    freq, gain = tsa.tsa_rotary_frequencies(tsa.TSA_ROTARY_WAVELENGTH, d, 500000.0, 8.0, 8192.0)
    cache = Cache(tsa, 3, max(lens) + steps, e4m3, 1)
    cu = np.concatenate([[0], np.cumsum(lens)])

    def step(qkv, positions, cu_q, kv_len):
        """One pass of a layer's attention over packed rows: rotate, keep, attend."""
        n = qkv.shape[0]
        Q, K, V = (qkv[:, a * d:b * d].unflatten(-1, (-1, d)) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
        row = qkv.stride(0)
        Qr, Kr, O = new(n, Hq, d), new(n, Hkv, d), new(n, Hq, d)
        strides = (0, d, row)
        rd = tsa.make_rotary_desc(1, Hq, Hkv, n, d, freq, gain=gain, q_strides=(n * row, d, row), k_strides=(n * row, d, row),
                                  q_out_strides=(n * Hq * d, d, Hq * d), k_out_strides=(n * Hkv * d, d, Hkv * d))
        view = lambda x: x.transpose(0, 1)[None]
        tsa.tsa_rotary(rd, view(Q), view(K), view(Qr), view(Kr), positions=positions[None])
        cd = cache.desc(n, v_strides=(row, d), max_q=int(max(np.diff(cu_q))))
        tsa.tsa_cache_write(cd, Kr, V, ints(cu_q), ints(kv_len), cache.table, *cache.pools, *cache.scales)
        tsa.tsa_attend_cache(cd, Qr, *cache.pools, ints(cu_q), ints(kv_len), cache.table, O, tsa.alloc_attend_cache_workspace(cd),
                             k_scales=cache.scales[0], v_scales=cache.scales[1])
        return Qr, Kr, V, O

    history = [[] for _ in lens]
    kv = list(lens)
    rows = gu.to_dev(gu.rand_bits(r, (T, (Hq + 2 * Hkv) * d)))
    pos = ints(np.concatenate([np.arange(n) for n in lens]))
    for s in range(1 + steps):
        cu_q = cu if s == 0 else np.arange(len(lens) + 1)
        Qr, Kr, V, O = step(rows, pos, cu_q, kv)
        L = max(kv)
        Kb, Vb = new(3, Hkv, L, d), new(3, Hkv, L, d)
        tsa.tsa_cache_read(cache.desc(0), *cache.pools, ints(kv), cache.table, L, Kb, Vb, *cache.scales)
        for i in range(len(lens)):
            cut = slice(cu_q[i], cu_q[i + 1])
            history[i].append((Kr[cut], V[cut]))
            K, Vi = (torch.cat([h[w] for h in history[i]]).transpose(0, 1).contiguous() for w in (0, 1))     # [Hkv, L, d]
            if e4m3:
                code = [srv.quantise_rows(gu.from_dev(x)) for x in (K, Vi)]
                K64, V64 = (srv.e4m3_value(c) * 2.0 ** (e[..., None].astype(float) - 127) for c, e in code)
            else:
                K64, V64 = (orc.bf16_to_f64(gu.from_dev(x)) for x in (K, Vi))
            # what reads back is what was kept
            assert np.array_equal(orc.bf16_to_f64(gu.from_dev(Kb[i, :, :kv[i]])), K64) and np.array_equal(orc.bf16_to_f64(gu.from_dev(Vb[i, :, :kv[i]])), V64)
            assert Kb[i, :, kv[i]:].abs().sum() == 0
            q, got = orc.bf16_to_f64(gu.from_dev(Qr[cut])), orc.bf16_to_f64(gu.from_dev(O[cut]))
            for h in range(Hq):
                g = h // (Hq // Hkv)
                want, _, mag = srv.attend(q[:, h], K64[g], V64[g], np.ones(kv[i], dtype=bool), d ** -0.5)
                assert (np.abs(got[:, h] - want) <= (2.0 ** -8 + 2.0 ** -12) * mag + 2.0 ** -8 * np.abs(want)).all(), (s, i, h)
        kv = [k + 1 for k in kv]
        rows = gu.to_dev(gu.rand_bits(r, (len(lens), (Hq + 2 * Hkv) * d)))
        pos = ints(np.array(kv) - 1)


def test_a_cached_prompt_through_the_prefill_entry_points(tsa):
    """One prompt: attention over the cache is tsa_attend's within rounding, and what the sparse layer makes of the cache read back is what it makes
    of the tensors that went into it, bit for bit."""
    r = np.random.Generator(np.random.PCG64(8100))
    L, k = 700, 200
    Q, K, V = (gu.to_dev(gu.rand_bits(r, (1, H, L, d))) for H in (Hq, Hkv, Hkv))
    cache = Cache(tsa, 1, L, 0, 2)
    cd = cache.desc(L, q_strides=(d, L * d), k_strides=(d, L * d), v_strides=(d, L * d), o_strides=(d, L * d))      # heads first
    packed = lambda x: x[0].transpose(0, 1)
    tsa.tsa_cache_write(cd, packed(K), packed(V), ints([0, L]), ints([L]), cache.table, *cache.pools)
    O, dense = new(1, Hq, L, d), new(1, Hq, L, d)
    lse, lse2 = new(L, Hq, dtype=torch.float32), new(1, Hq, L, dtype=torch.float32)
    tsa.tsa_attend_cache(cd, packed(Q), *cache.pools, ints([0, L]), ints([L]), cache.table, packed(O), tsa.alloc_attend_cache_workspace(cd), lse=lse)
    desc = tsa.make_desc(1, Hq, Hkv, L, d)
    tsa.tsa_attend(desc, Q, K, V, L, Hkv, dense, tsa.alloc_attend_workspace(desc, L, Hkv), lse=lse2)
    mag = np.stack([srv.attend(orc.bf16_to_f64(gu.from_dev(Q[0, h])), *(orc.bf16_to_f64(gu.from_dev(x[0, h // (Hq // Hkv)])) for x in (K, V)),
                               np.ones(L, dtype=bool), d ** -0.5)[2] for h in range(Hq)])
    err = (O[0].double() - dense[0].double()).abs().cpu().numpy()
    assert (err <= 2 * ((2.0 ** -8 + 2.0 ** -12) * mag + 2.0 ** -8 * mag)).all()           # each side is off by half of that at most
    assert (lse.T - lse2[0]).abs().max() <= 2.0 ** -11
    Kb, Vb = new(1, Hkv, L, d), new(1, Hkv, L, d)
    tsa.tsa_cache_read(cd, *cache.pools, ints([L]), cache.table, L, Kb, Vb)
    out = []
    for Kx, Vx in ((K, V), (Kb, Vb)):
        o, idx = new(1, Hq, L, d), new(1, Hq, k, dtype=torch.int32)
        tsa.tsa_forward(desc, Q, Kx, Vx, k, o, tsa.alloc_workspace(desc, k), idx_out=idx)
        out.append((o, idx))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


def test_a_captured_decoding_step(tsa):
    """Rotation, write and attention of one token per sequence in one graph; the lengths live on the device and grow there."""
    r = np.random.Generator(np.random.PCG64(8200))
    n, max_len = 4, 200
    freq, _ = tsa.tsa_rotary_frequencies(tsa.TSA_ROTARY_PLAIN, d, 10000.0)
    cache, eager = Cache(tsa, n, max_len, 1, 3), Cache(tsa, n, max_len, 1, 3)
    kv, cu = ints([1, 50, 16, 129]), ints(np.arange(n + 1))
    for c in (cache, eager):
        for p in c.pools:
            p.copy_(torch.from_numpy(np.random.Generator(np.random.PCG64(8)).integers(0, 100, tuple(p.shape)).astype(np.uint8)))
        for s in c.scales:
            s.fill_(122)
    Q, K, V, Qr, Kr, O = new(n, Hq, d), new(n, Hkv, d), new(n, Hkv, d), new(n, Hq, d), new(n, Hkv, d), new(n, Hq, d)
    pos = kv.clone()
    rd = tsa.make_rotary_desc(n, Hq, Hkv, 1, d, freq)          # a token per batch entry
    cd = cache.desc(n, max_q=1)
    ws, ws2 = tsa.alloc_attend_cache_workspace(cd), tsa.alloc_attend_cache_workspace(cd)
    one = lambda x: x[:, :, None]

    def step(c, ws):
        tsa.tsa_rotary(rd, one(Q), one(K), one(Qr), one(Kr), positions=pos[:, None])
        tsa.tsa_cache_write(cd, Kr, V, cu, kv, c.table, *c.pools, *c.scales)
        tsa.tsa_attend_cache(cd, Qr, *c.pools, cu, kv, c.table, O, ws, k_scales=c.scales[0], v_scales=c.scales[1])

    step(eager, ws2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cache, ws)
    step(cache, ws)                                        # (as eager had one)
    for _ in range(5):
        for x, H in ((Q, Hq), (K, Hkv), (V, Hkv)):
            x.copy_(gu.to_dev(gu.rand_bits(r, (n, H, d))))
        kv += 1
        pos.copy_(kv - 1)
        graph.replay()
        torch.cuda.synchronize()
        got = O.clone()
        O.fill_(3.0)
        step(eager, ws2)
        assert torch.equal(got, O)
        assert all(torch.equal(a, b) for a, b in zip(cache.pools + cache.scales, eager.pools + eager.scales))
