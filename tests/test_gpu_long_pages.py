"""Appending to and eviction from caches of the longest pages, through the C ABI, against plain fp64 forms."""
import pytest

from tests.test_gpu_paged import run_append, run_evict

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2406_18139_b200 import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("lens,new,hq,hkv,page", [([0, 1000], [1500, 40], 4, 2, 1024), ([65530, 9], [20, 1], 2, 1, 65536)])
def test_append(B, lens, new, hq, hkv, page):
    run_append(B, lens, new, hq, hkv, page)
    run_append(B, lens, new, hq, hkv, page, heads_first=False, interleaved=True, rotary=64)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("lens,budgets,windows,hkv,page", [([3000, 70], [1100, 60], [20, 70], 3, 1024), ([70000], [66000], [100], 1, 65536)])
def test_evict(B, in_place, lens, budgets, windows, hkv, page):
    run_evict(B, lens, budgets, windows, hkv, page, in_place)
