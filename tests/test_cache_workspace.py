"""What a call over the paged cache asks for as workspace, without a GPU: bounded whatever the number of sequences, and whatever the caller knows."""
import ctypes
import itertools

import pytest

from paper_2602_03216_amd import binding as tsa


def _bytes(n_seqs, n_tokens, max_q, keys, Hq=32, Hkv=8, d=128, fmt=0, window=0):
    desc = tsa.make_cache_desc(n_seqs, n_tokens, Hq, Hkv, d, 64, 1000, -(-keys // 64), fmt, max_q=max_q, window=window)
    return tsa.load_library().tsa_attend_cache_workspace_bytes(ctypes.byref(desc))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (28, 4), (8, 1), (32, 32), (4, 4)])
def test_bounded_for_any_number_of_sequences(Hq, Hkv, d):
    """Row tiles times parts stay below four times the 512 (768) places of the chip for workgroups of 128 rows (the most is three parts of a third more
    tiles than places), slots are less than twice the tiles and one a head more, a part of a tile is 128 rows of d + 2 floats; beside that what the
    shares of few rows leave, 17 MB at most."""
    bound = 2 * 4 * (768 if d == 64 else 512) * 128 * (d + 2) * 4 + Hkv * 4 * 128 * (d + 2) * 4 + 17.5e6
    for n, tokens, max_q, keys, fmt in itertools.product((1, 2, 64, 100, 1024, 4096), (1, 20, 32, 64, 272, 555, 2299, 6000), (0, 1, 17, 300), (2500, 16384, 131072),
                                                         (0, 1)):
        need = _bytes(n, tokens, max_q, keys, Hq, Hkv, d, fmt)
        assert 0 < need <= bound, (n, tokens, max_q, keys, fmt, need)


def test_tokens_of_a_caller_who_does_not_know_that_they_are_single():
    """64 of them took 1.1 GB, 4096 sequences with 32 of them 140 GB."""
    assert _bytes(64, 64, 1, 16384) < 10e6
    assert _bytes(64, 64, 0, 16384) < 100e6
    assert _bytes(4096, 32, 0, 131072) < 100e6
    assert _bytes(256, 272, 17, 16384) < 100e6


def test_a_size_that_is_refused_says_why():
    """Its own reason, not the one of the call before it."""
    lib = tsa.load_library()
    assert _bytes(1, 1, 1, 1000, d=80) == 0 and "head dimension 80" in tsa.tsa_last_error()
    big = tsa.make_cache_desc(1 << 19, 7, 32, 8, 128, 16, 10, 1 << 20)
    assert lib.tsa_attend_cache_workspace_bytes(ctypes.byref(big)) == 0 and "max_pages" in tsa.tsa_last_error()
    assert _bytes(1, 1, 1, 1000, d=80) == 0
    with pytest.raises(tsa.TsaError, match="max_pages"):
        tsa.alloc_attend_cache_workspace(big)
