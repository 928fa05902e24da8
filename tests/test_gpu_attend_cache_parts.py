"""tsa_attend_cache where the keys of prompts are cut into parts: more of them than the join takes at once, parts that start far into a long
context, each of the rules that choose their number."""
import copy
import ctypes

import numpy as np
import pytest
import torch

from tests.test_gpu_attend_cache import Batch, tsa  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def parts_of(tsa, desc):  # noqa: F811
    """Most parts of a row tile, from the size of what they leave: 128 rows of d + 2 floats for every slot, head and part, beside what the shares
    of few rows leave, which a call of single tokens needs too."""
    rows = desc.n_tokens * desc.Hq // desc.Hkv
    slots = rows // 128 + desc.n_seqs
    if desc.n_seqs > 1:
        slots = min(slots, 2 * rows // 129)
    need = tsa.load_library().tsa_attend_cache_workspace_bytes(ctypes.byref(desc))
    one = slots * desc.Hkv * 128 * (desc.d + 2) * 4
    single = tsa.make_cache_desc(desc.n_seqs, desc.n_seqs, desc.Hq, desc.Hkv, desc.d, desc.page_size, 1, desc.max_pages, desc.format, max_q=1)
    few = tsa.load_library().tsa_attend_cache_workspace_bytes(ctypes.byref(single))
    return max(1, round((need - few) / one))


def check_some(b, O, lse, heads):
    """Of the query heads `heads` alone."""
    g = b.Hq // b.Hkv
    some = copy.copy(b)
    some.Hq = some.Hkv = len(heads)
    some.scale = b.scale
    some.q = b.q[:, heads]
    some.rows = [(K[[h // g for h in heads]], V[[h // g for h in heads]], there) for K, V, there in b.rows]
    some.check(O[:, heads], lse[:, heads])


MANY = {
    "seventeen": (17, dict(new=[100], kv=[9000], Hq=1, Hkv=1, d=128, page=64)),
    "nine_and_gone": (9, dict(new=[70, 1, 130], kv=[5000, 300, 4700], Hq=2, Hkv=2, d=64, page=32, gone=[(0, 3), (0, 100), (2, 0), (2, 140), (2, 141)])),
    "windows": (23, dict(new=[129], kv=[12000], Hq=2, Hkv=1, d=128, page=16, window=5200)),
    "a_part_without_pages": (18, dict(new=[100], kv=[9000], Hq=2, Hkv=1, d=64, page=256, gone=[(0, p) for p in range(2, 9)])),
    "nothing_but_the_last_page": (18, dict(new=[90], kv=[9000], Hq=1, Hkv=1, d=64, page=256, gone=[(0, p) for p in range(35)])),
    "negative_positions": (17, dict(new=[300, 100], kv=[9000, 40], Hq=1, Hkv=1, d=64, page=64)),
}


@pytest.mark.parametrize("e4m3", [0, 1])
@pytest.mark.parametrize("name", list(MANY))
def test_more_parts_than_one_round_of_the_join(tsa, name, e4m3):  # noqa: F811
    most, c = MANY[name]
    b = Batch(8200 + list(MANY).index(name), e4m3=e4m3, **c)
    assert parts_of(tsa, b.desc(tsa)) == most
    first = b.run(tsa)
    b.check(*first)
    again = b.run(tsa)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


# 32 query heads on one KV head: a prompt of T tokens is T / 4 row tiles
RULES = {
    "as_many_as_run_at_once": (3, dict(new=[640], kv=[5000], d=128), 512),
    "two_rounds": (3, dict(new=[1270], kv=[5056], d=128), 512),
    "two_rounds_window": (3, dict(new=[1270], kv=[9000], d=128, window=3900), 512),
    "three_of_a_few_more": (3, dict(new=[2110], kv=[8200], d=128), 512),
    "three_of_a_few_more_d64": (3, dict(new=[3150], kv=[8200], d=64), 768),
    "two_rounds_d64": (3, dict(new=[2000], kv=[5000], d=64), 768),
    "one_round": (1, dict(new=[2000], kv=[4000], d=128), 512),
}


@pytest.mark.parametrize("name,e4m3", [(n, e) for n, r in RULES.items() for e in (0, 1) if not (e and r[2] == 768)])      # (d = 64 in 8 bits has 512 places)
def test_every_rule_for_the_parts(tsa, name, e4m3):  # noqa: F811
    most, c, _ = RULES[name]
    b = Batch(8300 + list(RULES).index(name), Hq=32, Hkv=1, page=64, e4m3=e4m3, gone=[(0, 7), (0, 40)], **c)
    assert parts_of(tsa, b.desc(tsa)) == most
    O, lse = b.run(tsa)
    check_some(b, O, lse, [0, 13, 31])
    assert np.isfinite(lse.cpu().numpy()).all()


@pytest.mark.parametrize("new,kv,d,e4m3,window", [(1270, 2560, 128, 0, 0), (1270, 2560, 64, 1, 0), (2110, 2560, 128, 0, 0), (2110, 2560, 128, 1, 0), (1270, 3840, 128, 0, 1200),
                                                  (1270, 5120, 128, 0, 0), (3150, 3200, 64, 0, 0)])
def test_a_wide_table_over_short_contexts(tsa, new, kv, d, e4m3, window):  # noqa: F811
    """A prompt's parts go by its length: a table of as many pages as a model can have and one that ends with the context give the same bits."""
    b = Batch(8400 + new + d, [new], [kv], 32, 1, d, 64, e4m3=e4m3, window=window)
    want = b.run(tsa)
    check_some(b, *want, [5])
    b.tab = np.pad(b.tab, ((0, 0), (0, 2048 - b.max_pages)), constant_values=-1)
    b.max_pages = 2048
    got = b.run(tsa)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
