"""Appending to a paged cache and eviction from it, through the C ABI, against plain fp64 forms.

Tolerance of normed and rotated rows: a value is a sum of two products of fp32 numbers, each within some ten
roundings (2^-24) of its fp64 value, and is rounded to bf16 once (half a step: 2^-8 of the value), so
|got - ref| <= 2^-8 |ref| + 4e-6 (|a| + |b|), with |a| + |b| at most twice the row's largest normed value.
What is only moved is equal bit for bit.
"""
import math

import pytest
import torch

from tests.paged import Cache, D, kept64, norm_rotate64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2406_18139_b200 import binding
    binding.lib()
    return binding


def same(a, b):
    """Equal bit for bit, NaN included."""
    kind = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


def freqs(rotary, theta=10000.0):
    return [theta ** (-2.0 * i / rotary) for i in range(rotary // 2)]


# ---- appending ---------------------------------------------------------------------------------------

def run_append(B, lens, new, hq, hkv, page, norm=True, rotary=128, interleaved=False, heads_first=True, far=0, in_place=False,
               strided=False, with_q=True, seed=1):
    c = Cache(lens, hkv, page, seed, heads_first, room=max(new))
    total, cu = sum(new), [sum(new[:i]) for i in range(len(new) + 1)]
    if strided:                                   # one buffer of q, k and v, as a fused projection leaves it
        qkv = (c.normal(total, hq + 2 * hkv, D) * 3).bfloat16()
        q, k, v = qkv.split([hq, hkv, hkv], dim=1)
    else:
        q, k, v = ((c.normal(total, h, D) * 3).bfloat16() for h in (hq, hkv, hkv))
    qw, kw = ((1 + c.normal(D)).bfloat16() if norm else None for _ in range(2))
    pos = (torch.cat([torch.arange(a, a + n) for a, n in zip(lens, new)]) + far).int().cuda() if rotary else None
    inv = freqs(rotary) if rotary else []
    if not with_q:
        q = None
    q_in = None if q is None else q.clone()
    q_out = None if q is None else q if in_place else torch.full((total, hq, D), math.nan, dtype=torch.bfloat16, device="cuda")
    paged = B.make_paged_layout(q_out, c.k, c.table, n_q_heads=hq)
    ws = B.alloc_paged_workspace(paged, new, [a + b for a, b in zip(lens, new)])
    opt = B.make_append_options(qw, kw, 1e-6, inv, interleaved) if norm or rotary else None
    want_k, want_v, want_m = c.k.clone(), c.v.clone(), c.mass.clone()
    k64 = norm_rotate64(k, kw, 1e-6, pos, inv, interleaved)
    B.check(B.lookm_append_rows(q, k, v, pos, cu, lens, B.make_layout(q_in if q is None else q, k), opt, q_out, c.k, c.v, c.mass, c.table,
                                paged, ws))
    B.check(B.lookm_device_status(ws))
    row_max = lambda x: x.abs().amax(-1, keepdim=True)
    for r, (a, n) in enumerate(zip(lens, new)):
        if not n:
            continue
        p, o = c.where(r, a, n)
        got, ref = c.k[p, :, o].double(), k64[cu[r]:cu[r + 1]]
        assert ((got - ref).abs() <= 2 ** -8 * ref.abs() + 8e-6 * row_max(ref)).all()
        assert same(c.v[p, :, o], v[cu[r]:cu[r + 1]])
        assert (c.mass[p, :, o] == 0).all()
        want_k[p, :, o], want_v[p, :, o], want_m[p, :, o] = c.k[p, :, o], c.v[p, :, o], 0.0
    # every other row of the pools is as it was
    assert same(c.k, want_k) and same(c.v, want_v) and same(c.mass, want_m)
    if q is not None:
        ref = norm_rotate64(q_in, qw, 1e-6, pos, inv, interleaved)
        assert ((q_out.double() - ref).abs() <= 2 ** -8 * ref.abs() + 8e-6 * row_max(ref)).all()
        if not norm and not rotary:
            assert same(q_out, q_in)


@pytest.mark.parametrize("lens,new,hq,hkv,page", [([0], [1], 1, 1, 16), ([15], [1], 4, 2, 16), ([16], [1], 32, 8, 16),
                                                  ([0], [700], 32, 32, 16), ([100, 0, 7], [3, 0, 129], 6, 2, 32),
                                                  ([0, 0, 0], [0, 5, 0], 5, 1, 64), ([1000], [333], 40, 40, 128),
                                                  ([63] * 20, [2] * 20, 8, 8, 64), ([17] * 130, [1] * 129 + [40], 3, 1, 16)])
def test_append_places_normed_and_rotated_rows(B, lens, new, hq, hkv, page):
    run_append(B, lens, new, hq, hkv, page, seed=len(lens))


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("rotary,interleaved", [(0, False), (16, False), (48, True), (64, False), (64, True), (112, False),
                                                (128, True), (128, False)])
def test_append_kinds_of_rotation(B, norm, rotary, interleaved):
    run_append(B, [5, 30], [37, 4], 6, 3, 16, norm, rotary, interleaved, heads_first=rotary % 32 == 0)


@pytest.mark.parametrize("kw", [dict(far=1 << 20), dict(far=(1 << 31) - 2000), dict(far=-50), dict(in_place=True), dict(strided=True),
                                dict(strided=True, in_place=True), dict(with_q=False), dict(with_q=False, norm=False, rotary=0),
                                dict(norm=False, rotary=0), dict(heads_first=False)])
def test_append_positions_strides_and_queries_in_place(B, kw):
    run_append(B, [100, 3], [41, 18], 8, 2, 32, **kw)


def test_append_reports_a_bad_page_and_writes_nothing_there(B):
    c = Cache([10, 10], 2, 16, 5, room=30)
    c.table[1, 1] = 10 ** 6
    k, v = (c.normal(60, 2, D).bfloat16() for _ in range(2))
    paged = B.make_paged_layout(None, c.k, c.table, n_q_heads=2)
    ws = B.alloc_paged_workspace(paged, [30, 30], [40, 40])
    want = c.k.clone()
    lay = B.make_layout(None, k)
    B.check(B.lookm_append_rows(None, k, v, None, [0, 30, 60], [10, 10], lay, None, None, c.k, c.v, None, c.table, paged, ws))
    assert B.lookm_device_status(ws) == B.ERR_DEVICE_BAD_INDEX
    assert B.lookm_device_status(ws) == B.OK
    for r, first, n, tok in ((0, 10, 30, 0), (1, 10, 6, 30), (1, 32, 8, 52)):
        p, o = c.where(r, first, n)
        want[p, :, o] = k[tok:tok + n]
    assert same(c.k, want)


# ---- eviction --------------------------------------------------------------------------------------------

def run_evict(B, lens, budgets, windows, hkv, page, in_place, mass=None, heads_first=True, seed=3, with_kept=True):
    c = Cache(lens, hkv, page, seed, heads_first)
    if mass is not None:
        for r, n in enumerate(lens):
            c.put(c.mass, r, 0, mass(n, hkv))
    old = c.k.clone(), c.v.clone(), c.mass.clone()
    if in_place:
        ok, ov, om, table = c.k, c.v, c.mass, c.table
    else:
        perm = torch.randperm(len(c.k), generator=c.gen).int().cuda()
        table = torch.where(c.table >= 0, perm[c.table.clamp(min=0).long()], -7).int()
        ok, ov, om = c.k.clone(), c.v.clone(), c.mass.clone()
    want = ok.clone(), ov.clone(), om.clone()
    keep = [min(b, n) for b, n in zip(budgets, lens)]
    kept = torch.full((hkv * sum(keep) + 1,), -3, dtype=torch.int32, device="cuda") if with_kept else None
    paged = B.make_paged_layout(None, c.k, c.table, n_q_heads=hkv)
    ws = B.alloc_paged_workspace(paged, None, lens)
    B.check(B.lookm_evict(c.k, c.v, c.mass, c.table, lens, budgets, windows, paged, ok, ov, om, table, kept, ws))
    B.check(B.lookm_device_status(ws))
    at = 0
    for r, n in enumerate(lens):
        if not keep[r]:
            continue
        m = c.rows(old[2], r, n).t().cpu().tolist()
        to, off = c.where(r, 0, keep[r], table)
        for h in range(hkv):
            ref = kept64(m[h], budgets[r], windows[r])
            if with_kept:
                assert kept[at:at + keep[r]].tolist() == ref, (r, h)
            at += keep[r]
            idx = torch.tensor(ref, device="cuda")
            src, soff = c.table[r].long()[idx // page], idx % page
            for o, w in zip(old, want):
                w[to, h, off] = o[src, h, soff]
    assert not with_kept or int(kept[-1]) == -3
    assert all(same(a, b) for a, b in zip((ok, ov, om), want))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("lens,budgets,windows,hkv,page", [
    ([1], [1], [0], 1, 16), ([2], [1], [0], 1, 16), ([2], [1], [1], 1, 16), ([17], [16], [4], 3, 16), ([100], [100], [10], 2, 32),
    ([100], [999], [10], 2, 32), ([700], [140], [16], 4, 16), ([700], [140], [140], 4, 16), ([700], [140], [500], 4, 64),
    ([33, 0, 500], [20, 5, 499], [3, 1, 8], 5, 16), ([8192], [1638], [32], 8, 16), ([2048, 2049], [2047, 1], [0, 0], 2, 128),
    ([5000, 1200, 37], [4000, 960, 29], [32, 32, 32], 32, 64), ([33000], [30000], [64], 2, 64), ([40000], [9000], [7], 1, 256), ([300000], [100000], [33], 1, 256),
    ([36000, 50], [1000, 49], [9, 9], 80, 64),
    ([40] * 131, [20] * 131, [2] * 131, 2, 16)])
def test_evict_keeps_the_heaviest_rows(B, in_place, lens, budgets, windows, hkv, page):
    run_evict(B, lens, budgets, windows, hkv, page, in_place, seed=sum(lens), heads_first=hkv % 2 == 0)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind", ["all equal", "few values", "signs and zeros", "infinities and nan", "denormal"])
def test_evict_ties_and_odd_masses(B, in_place, kind):
    def mass(n, h):
        x = torch.randint(0, 3, (n, h), generator=torch.Generator().manual_seed(n)).float().cuda()
        if kind == "all equal":
            return x * 0 + 2.5
        if kind == "few values":
            return x
        if kind == "signs and zeros":
            return torch.where(x == 0, -0.0, x - 1)
        if kind == "denormal":
            return x * 1e-42
        return torch.where(x == 0, math.nan, torch.where(x == 1, math.inf, -math.inf))

    run_evict(B, [300, 41], [170, 20], [16, 3], 3, 16, in_place, mass)


def test_evict_without_a_list_and_with_pages_that_are_no_pages(B):
    run_evict(B, [300], [170], [16], 3, 16, True, with_kept=False)
    c = Cache([100], 2, 16, 9)
    c.table[0, 2] = len(c.k)
    paged = B.make_paged_layout(None, c.k, c.table, n_q_heads=2)
    ws = B.alloc_paged_workspace(paged, None, [100])
    other = torch.zeros_like(c.k), torch.zeros_like(c.v), torch.zeros_like(c.mass)
    table = torch.arange(8, dtype=torch.int32, device="cuda")[None]
    B.check(B.lookm_evict(c.k, c.v, c.mass, c.table, [100], [50], [60], paged, *other, table, None, ws))
    assert B.lookm_device_status(ws) == B.OK                      # rows 32 to 47 are neither read nor kept: the window is all
    B.check(B.lookm_evict(c.k, c.v, c.mass, c.table, [100], [90], [4], paged, *other, table, None, ws))
    assert B.lookm_device_status(ws) == B.ERR_DEVICE_BAD_INDEX
