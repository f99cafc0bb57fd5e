"""Attention over a paged cache in each of the plans by which a call's work is divided (whole units or equal shares, sets of one or of two
query tiles), through the C ABI, against fp64.  Tolerances: those of the single operators' tests."""
import math

import pytest
import torch

from tests.chunk_plan import Plan
from tests.paged import D
from tests.test_gpu_chunk import run_chunk

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2406_18139_b200 import binding
    binding.lib()
    return binding


def plan_of(new, lens, hq, hkv, page):
    return Plan(new, lens, hq, hkv, page, torch.cuda.get_device_properties(0).multi_processor_count)


def rising(c, q):
    """A change of cache and queries by which the largest logit of a tile of 128 rows is some seven above that of the tile before it, more than
    the reference puts up with (8 bits); after nine tiles they begin anew."""
    for r, length in enumerate(c.lens):
        k = c.rows(c.k, r, length).float()
        k[..., 0] = (torch.arange(length, device="cuda") // 128 % 9)[:, None]
        c.put(c.k, r, 0, k)
    q[..., 0] = 80.0


@pytest.mark.parametrize("n,new,hq,hkv,page,shares", [(800, 1, 8, 8, 64, False), (1200, 17, 8, 2, 16, False), (700, 700, 4, 4, 32, False),
                                                      (9000, 3, 32, 8, 16, True), (9000, 300, 8, 2, 64, True)])
def test_two_streams_of_one_query_tile_both_rescaled(B, n, new, hq, hkv, page, shares):
    """Stream 0 adds up outputs that stream 1 has rescaled just before: every tile's maximum lies above the last one's."""
    p = plan_of([new], [n], hq, hkv, page)
    assert p.launches[0]["pairs"] == 0 and p.launches[0]["shares"] == shares
    run_chunk(B, [n], [new], hq, hkv, page, change=rising, seed=n)
    assert B.lookm_last_launch_count() == p.n_launches()


@pytest.mark.parametrize("page", [16, 64])
def test_infinities_in_many_short_items(B, page):
    """Pairs of query tiles and single ones of one tile of cached rows, several to a CTA, each with an infinity that only its last rows see."""
    lens = [128] * 40 + [20 + i % 44 for i in range(200)]
    p = plan_of(lens, lens, 8, 4, page)
    assert len(p.launches) == 2 and p.launches[0]["units"] > 3 * 128 and p.launches[0]["pairs"] == 160
    assert not any(x["shares"] for x in p.launches)

    def change(c, q):
        for r, n in enumerate(lens):
            v = c.rows(c.v, r, n).float()
            v[n - 1 - r % 7, r % 4, r % 128] = math.inf if r % 3 else math.nan
            c.put(c.v, r, 0, v)

    run_chunk(B, lens, lens, 8, 4, page, change=change)
    assert B.lookm_last_launch_count() == p.n_launches()
