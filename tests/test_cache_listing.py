"""The kernels of the attention over the cache as they are built, read as assembly without a GPU: which ones there are, and the wait states in front
of their loads into LDS."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2602_03216_amd import build
from tests import test_load_to_lds as listing
from tests.test_load_to_lds import hipcc  # noqa: F401  (the fixture)


@pytest.fixture(scope="module")
def kernels(hipcc):  # noqa: F811
    """(name, arguments of its template as text) -> its lines"""
    files = ["attend_cache.hip", "attend_cache_many.hip"]
    with ThreadPoolExecutor(len(files)) as pool:
        parts = pool.map(lambda f: listing._assembly(os.path.join(listing.CSRC, f), build.EXTRA[f]), files)
    code = {name: lines for part in parts for name, lines in part.items()}
    plain = subprocess.run(["c++filt"], input="\n".join(code), capture_output=True, text=True, check=True).stdout.splitlines()
    out = {}
    for name, lines in zip(plain, code.values()):
        found = re.search(r"::(\w+)<([^>]*)>\(", name)
        if found:
            out[found[1], tuple(found[2].split(", "))] = lines
    return out


def test_every_kernel_is_one_that_a_call_can_reach(kernels):
    both = [(d, e) for d in ("64", "128") for e in ("false", "true")]
    few = {(d, e, mb, "true") for d, e in both for mb in ("1", "2", "4")} | {(d, e, "1", "false") for d, e in both}
    few -= {("128", "true", "4", "true")}                   # 33 to 64 rows in 8 bits at d = 128 are two tiles of 32 ...
    few |= {("128", "true", "2", "false")}                  # ... whose keys the other one reads again
    assert {k[1] for k in kernels if k[0] == "attend_few_rows"} == few
    assert {k[1] for k in kernels if k[0] == "attend_whole_tiles"} == set(both)
    assert {k[1] for k in kernels if k[0] == "attend_many_rows"} == {(*x, f) for x in both for f in ("false", "true")}
    assert {k[1] for k in kernels if k[0] in ("join_few_rows", "join_many_rows")} == {("64",), ("128",)}


def _loads_to_lds(code):
    return [i for i, line in enumerate(code) if line.startswith("global_load_lds")]


def test_every_load_to_lds_has_its_wait_states(kernels, monkeypatch):
    """Five between a vector instruction that wrote m0 or the scalar base of a load and the load, which is inline assembly that the compiler's own hazard
    pass does not look into (its vector address needs none)."""
    monkeypatch.setattr(listing, "_loads", _loads_to_lds)
    for (name, args), code in kernels.items():
        if not name.startswith("attend"):
            continue
        few = name != "attend_many_rows" or args[2] == "true"
        # (8 bits with many rows pass the registers)
        assert len(_loads_to_lds(code)) >= (4 if few or args[1] == "false" else 0), (name, args)
        assert not listing._short_waits(code), (name, args, listing._short_waits(code)[:3])


def test_the_search_sees_these_loads(monkeypatch):
    """on listings made up here"""
    monkeypatch.setattr(listing, "_loads", _loads_to_lds)
    plain, based = "global_load_lds_dwordx4 v[2:3], off nt", "global_load_lds_dwordx4 v2, s[4:5]"
    assert listing._short_waits(["v_readfirstlane_b32 m0, v2", "s_nop 3", plain]) and listing._short_waits(["v_readlane_b32 s5, v2, 1", "s_nop 0", based])
    assert not listing._short_waits(["v_readfirstlane_b32 m0, v2", "s_nop 4", plain]) and not listing._short_waits(["v_readlane_b32 s5, v2, 1", plain])
