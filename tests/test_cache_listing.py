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
