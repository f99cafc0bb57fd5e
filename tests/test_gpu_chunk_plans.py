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


def run(B, lens, new, hq, hkv, page, want, change=None, **kw):
    """`want`: what every launch of the plan has."""
    p = plan_of(new, lens, hq, hkv, page)
    got = [dict(shares=x["shares"], pairs=x["pairs"] > 0) for x in p.launches]
    assert got == want, p.launches
    run_chunk(B, lens, new, hq, hkv, page, change=change, seed=sum(lens), **kw)
    assert B.lookm_last_launch_count() == p.n_launches()
    return p


WHOLE_PAIRS, WHOLE_ONES = dict(shares=False, pairs=True), dict(shares=False, pairs=False)
CUT_PAIRS, CUT_ONES = dict(shares=True, pairs=True), dict(shares=True, pairs=False)


@pytest.mark.parametrize("lens,new,hq,hkv,page", [([2600], [2600], 16, 16, 128), ([1300], [1300], 32, 32, 64), ([900] * 2, [900] * 2, 64, 32, 32),
                                                  ([1200, 1500, 2100], [1200] * 3, 32, 32, 16)])
@pytest.mark.parametrize("rises", [False, True])
def test_more_whole_pairs_than_sms(B, lens, new, hq, hkv, page, rises):
    """What a long prompt is made of: several rounds of the deal, one pair of query tiles after another on a CTA.  With maxima that rise from tile to
    tile, so that outputs are rescaled, and with ones that don't."""
    p = run(B, lens, new, hq, hkv, page, [WHOLE_PAIRS], rising if rises else None)
    assert p.launches[0]["units"] > torch.cuda.get_device_properties(0).multi_processor_count


@pytest.mark.parametrize("n,new,hq,hkv,page,want", [(20000, 300, 16, 4, 32, CUT_PAIRS), (12000, 300, 16, 4, 32, CUT_ONES),
                                                    (9000, 20, 8, 2, 16, CUT_ONES), (1024, 1024, 32, 32, 64, WHOLE_ONES)])
@pytest.mark.parametrize("rises", [False, True])
def test_the_other_plans(B, n, new, hq, hkv, page, want, rises):
    run(B, [n], [new], hq, hkv, page, [want], rising if rises else None)


@pytest.mark.parametrize("new,step,hq,want", [(1, 400, 2, [CUT_ONES, CUT_ONES]), (150, 400, 1, [CUT_PAIRS, CUT_PAIRS]), (3, 10, 2, [WHOLE_ONES] * 2)])
def test_a_batch_of_more_entries_than_a_launch_takes(B, new, step, hq, want):
    """In shares both launches use the same memory for the pieces."""
    first = {1: 9000, 150: 3000, 3: 200}[new]
    run(B, [first + step * (i % 9) for i in range(140)], [new] * 140, hq, 1, 32, want)


@pytest.mark.parametrize("n,new,hq,hkv,page,want", [(3000, 40, 4, 2, 1024, CUT_ONES), (70000, 200, 2, 1, 65536, CUT_ONES),
                                                    (70000, 1, 2, 1, 65536, CUT_ONES), (300, 300, 2, 2, 65536, WHOLE_PAIRS)])
def test_long_pages(B, n, new, hq, hkv, page, want):
    run(B, [n], [new], hq, hkv, page, [want], heads_first=n % 2 == 0)


@pytest.mark.parametrize("n,new,hq,hkv,page,want,loaders", [
    (9000, 20, 8, 2, 16, CUT_ONES, 2), (200, 20, 8, 2, 16, WHOLE_ONES, 2), (9000, 300, 8, 2, 64, CUT_ONES, 1), (20000, 300, 16, 4, 32, CUT_PAIRS, 1),
    (1300, 1300, 32, 32, 64, WHOLE_PAIRS, 1)])
@pytest.mark.parametrize("kind", ["v nan last", "v inf", "k nan last", "k -inf", "k all -inf"])
def test_infinities_and_nan_in_every_plan(B, n, new, hq, hkv, page, want, loaders, kind):
    """In pieces of units, and where one warp alone looks the values over."""
    def change(c, q):
        k, v = c.rows(c.k, 0, n).float(), c.rows(c.v, 0, n).float()
        if kind == "v nan last":
            v[n - 1, 0, 5] = math.nan
        elif kind == "v inf":
            v[n - 1, -1, 0], v[n - (new + 1) // 2, 0, 77], v[n - (new + 1) // 2, 0, 78] = math.inf, -math.inf, math.inf
            v[max(0, n - new - 3), 0, 3] = math.inf
        elif kind == "k nan last":
            k[n - 1, 0, 9] = math.nan
        else:
            q[..., 4] = 1.0
            if kind == "k -inf":
                k[n - 1, :, 4] = -math.inf
                k[n // 2, 0, 4] = -math.inf
            else:
                k[:, 0, 4] = -math.inf
        c.put(c.k, 0, 0, k)
        c.put(c.v, 0, 0, v)

    p = run(B, [n], [new], hq, hkv, page, [want], change)
    assert p.loaders == loaders


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
