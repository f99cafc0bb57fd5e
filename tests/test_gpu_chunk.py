"""Attention over a paged cache (chunks of new tokens, and single ones with their weights), through the C ABI, against fp64.

Tolerances.  Products of bf16 are exact in fp32; a logit is a sum of 128 of them whose roundings (2^-24 of the partial
sums each, or cut off) stay below e = 2^-17 of sum |q_d k_d| * scale for 128 terms; exponentials, their argument's and the log-sum-exp's own
roundings add less than 4e-6 (1 + |lse|) for |lse| up to some tens.  So
  lse     |got - ref| <= e + 4e-6 (1 + |lse|)
  weights a relative error of twice that
  out     every probability is rounded to bf16 (2^-8 of it at most) and so is the result:
          2^-8 (|ref| + sum w |v|) + the weights' error times sum w |v|
Rows behind a cache's end and pages of nobody hold NaN throughout.
"""
import math

import pytest
import torch

from tests.paged import Cache, D, attention64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2406_18139_b200 import binding
    binding.lib()
    return binding


def reference(c, r, q, n_new, scale):
    """fp64 results of a request and what they may be off: out, lse, weights, tolerances of these three."""
    n, k, v = c.lens[r], c.rows(c.k, r, c.lens[r]), c.rows(c.v, r, c.lens[r])
    out, lse, w = attention64(q, k, v, n - n_new, scale)
    g = q.shape[1] // k.shape[1]
    kk, vv = (x.double().abs().nan_to_num(0, 0, 0).repeat_interleave(g, dim=1).transpose(0, 1) for x in (k, v))
    e = 2.0 ** -17 * torch.matmul(q.double().abs().transpose(0, 1), kk.transpose(1, 2)).amax(-1) * scale
    tol_lse = e + 4e-6 * (1 + lse.abs())
    size = torch.matmul(w.nan_to_num(0, 0, 0), vv).transpose(0, 1)
    tol_out = 2.0 ** -8 * (out.abs() + size) + 2 * tol_lse.t()[..., None] * size
    return out, lse, w, tol_out, tol_lse, 2 * tol_lse[..., None] * w


def close(got, ref, tol):
    """Within tol where ref is finite, the same infinity or NaN where not."""
    got, fine = got.double(), torch.isfinite(ref)
    odd = torch.where(torch.isnan(ref), torch.isnan(got), got == ref)
    return torch.where(fine, (got - ref).abs() <= tol, odd).all()


def run_chunk(B, lens, new, hq, hkv, page, heads_first=True, scale=0.0, q_scale=1.0, strided=False, want_lse=True, change=None, seed=1):
    """Returns nothing, asserts.  `change(c, q)` may alter the cache or the queries first."""
    c = Cache(lens, hkv, page, seed, heads_first)
    total, cu = sum(new), [sum(new[:i]) for i in range(len(new) + 1)]
    q = (c.normal(max(total, 1), (2 if strided else 1) * hq, D) * q_scale).bfloat16()[:, :hq]
    if change:
        change(c, q)
    out = torch.full((total + 1, hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((hq * total + 1,), 7.0, device="cuda") if want_lse else None
    paged = B.make_paged_layout(q, c.k, c.table, scale)
    ws = B.alloc_paged_workspace(paged, new, lens)
    ws[256:] = 255                                # NaN: nothing may be taken from an earlier call
    before = c.k.clone(), c.v.clone()
    B.check(B.lookm_chunk_attention(q, c.k, c.v, c.table, cu, lens, paged, out, lse, ws))
    B.check(B.lookm_device_status(ws))
    for a, b in zip(before, (c.k, c.v)):
        assert torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))
    assert (out[total] == 7).all() and (lse is None or lse[-1] == 7)
    sc = scale or D ** -0.5
    for r, n in enumerate(new):
        if not n:
            continue
        mine = slice(cu[r], cu[r + 1])
        ref, ref_lse, _, tol, tol_lse, _ = reference(c, r, q[mine], n, sc)
        assert close(out[mine], ref, tol), (r, float(((out[mine].double() - ref).abs() / tol).max()))
        if want_lse:
            assert close(lse[:-1].view(hq, total)[:, mine], ref_lse, tol_lse), r
    again = torch.empty_like(out)
    B.check(B.lookm_chunk_attention(q, c.k, c.v, c.table, cu, lens, paged, again, None, ws))
    B.check(B.lookm_device_status(ws))
    assert torch.equal(out[:total].view(torch.int16), again[:total].view(torch.int16))


@pytest.mark.parametrize("n,new,hq,hkv,page", [(1, 1, 1, 1, 16), (2, 2, 1, 1, 16), (16, 1, 4, 1, 16), (17, 17, 2, 2, 16), (127, 127, 1, 1, 32),
                                               (128, 128, 1, 1, 128), (129, 129, 2, 1, 64), (129, 1, 8, 8, 16), (256, 129, 1, 1, 16),
                                               (255, 200, 3, 1, 32), (300, 257, 2, 2, 256), (640, 130, 4, 2, 16), (700, 700, 4, 4, 64),
                                               (1000, 3, 32, 8, 16), (1025, 1025, 1, 1, 128), (2000, 37, 7, 1, 32), (511, 64, 10, 2, 16),
                                               (400, 5, 64, 1, 16), (385, 4, 128, 1, 16), (200, 2, 127, 1, 64), (9000, 1, 8, 2, 64),
                                               (5000, 260, 6, 2, 16)])
def test_one_request(B, n, new, hq, hkv, page):
    run_chunk(B, [n], [new], hq, hkv, page, heads_first=n % 2 == 0, seed=n)


@pytest.mark.parametrize("lens,new,hq,hkv,page", [
    ([5, 300, 129], [1, 0, 129], 4, 2, 16), ([0, 40], [0, 40], 2, 2, 32), ([700, 3, 2500], [200, 3, 1], 8, 2, 16),
    ([1000] * 20, [1] * 20, 8, 8, 64), ([100, 90, 80] * 50, [1, 20, 0] * 50, 2, 1, 16), ([4096, 17, 1300, 6000], [300, 17, 2, 128], 16, 4, 128),
    ([3000, 2000], [1500, 1999], 5, 5, 32)])
def test_ragged_batches(B, lens, new, hq, hkv, page):
    run_chunk(B, lens, new, hq, hkv, page, seed=len(lens))


@pytest.mark.parametrize("kw", [dict(scale=0.3), dict(q_scale=6.0), dict(q_scale=0.0), dict(strided=True), dict(want_lse=False),
                                dict(heads_first=False)])
def test_scales_and_strides(B, kw):
    run_chunk(B, [900, 33], [140, 2], 8, 2, 16, **kw)


@pytest.mark.parametrize("new", [1, 150, 600])
def test_logits_that_grow_along_the_rows(B, new):
    """The maximum rises in every tile, by more than the reference puts up with."""
    def change(c, q):
        k = c.rows(c.k, 0, 900).float()
        ramp = torch.linspace(0, 40, 900, device="cuda")[:, None]
        k[..., 0] = ramp
        q[..., 0] = 12.0
        c.put(c.k, 0, 0, k)

    run_chunk(B, [900], [new], 4, 2, 32, change=change)


@pytest.mark.parametrize("n,new,hq,hkv", [(300, 150, 4, 2), (1000, 40, 8, 2), (700, 700, 2, 2), (129, 1, 4, 4)])
@pytest.mark.parametrize("kind", ["v nan last", "v inf", "k nan last", "k inf", "k all -inf"])
def test_infinities_and_nan_stay_with_the_rows_that_see_them(B, n, new, hq, hkv, kind):
    def change(c, q):
        k, v = c.rows(c.k, 0, n).float(), c.rows(c.v, 0, n).float()
        if kind == "v nan last":
            v[n - 1, 0, 5] = math.nan
        elif kind == "v inf":
            v[n - 1, -1, 0], v[n - (new + 1) // 2, 0, 77], v[n - (new + 1) // 2, 0, 78] = math.inf, -math.inf, math.inf
            v[max(0, n - new - 3), 0, 3] = math.inf
        elif kind == "k nan last":
            k[n - 1, 0, 9] = math.nan
        elif kind == "k inf":
            q[..., 4] = 1.0
            k[n - 1, :, 4] = -math.inf
            k[n // 2, 0, 4] = -math.inf
        else:
            q[..., 4] = 1.0
            k[:, 0, 4] = -math.inf
        c.put(c.k, 0, 0, k)
        c.put(c.v, 0, 0, v)

    run_chunk(B, [n], [new], hq, hkv, 16, change=change)


def test_a_bad_page_is_reported_and_reads_as_zeros(B):
    c = Cache([100], 2, 16, 4)
    c.put(c.k, 0, 32, c.normal(16, 2, D) * 0)
    c.put(c.v, 0, 32, c.normal(16, 2, D) * 0)
    q = c.normal(3, 4, D).bfloat16()
    paged = B.make_paged_layout(q, c.k, c.table)
    ws = B.alloc_paged_workspace(paged, [3], [100])
    out, bad = (torch.empty(3, 4, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.check(B.lookm_chunk_attention(q, c.k, c.v, c.table, [0, 3], [100], paged, out, None, ws))
    assert B.lookm_device_status(ws) == B.OK
    c.table[0, 2] = -1
    B.check(B.lookm_chunk_attention(q, c.k, c.v, c.table, [0, 3], [100], paged, bad, None, ws))
    assert B.lookm_device_status(ws) == B.ERR_DEVICE_BAD_INDEX
    assert torch.equal(out, bad)


def run_step(B, lens, hq, hkv, page, want_lse=True, q_scale=1.0, seed=1, heads_first=True):
    c = Cache(lens, hkv, page, seed, heads_first)
    n = len(lens)
    q = (c.normal(n, hq, D) * q_scale).bfloat16()
    out = torch.full((n, hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((hq, n), 7.0, device="cuda") if want_lse else None
    paged = B.make_paged_layout(q, c.k, c.table)
    ws = B.alloc_paged_workspace(paged, None, lens)
    ws[256:] = 255
    old = c.mass.clone()
    want = old.clone()
    B.check(B.lookm_step_attention(q, c.k, c.v, c.mass, c.table, lens, paged, out, lse, ws))
    B.check(B.lookm_device_status(ws))
    for r, k in enumerate(lens):
        ref, ref_lse, w, tol, tol_lse, tol_w = reference(c, r, q[r:r + 1], 1, D ** -0.5)
        assert close(out[r:r + 1], ref, tol), (r, float(((out[r:r + 1].double() - ref).abs() / tol).max()))
        if want_lse:
            assert close(lse[:, r:r + 1], ref_lse, tol_lse)
        p, o = c.where(r, 0, k)
        sums, tols = (x[:, 0].view(hkv, hq // hkv, k).sum(1).t() for x in (w, tol_w))
        ref_m = old[p, :, o].double() + sums
        assert ((c.mass[p, :, o].double() - ref_m).abs() <= tols + 2.0 ** -23 * (hq // hkv + 1) * ref_m.abs()).all(), r
        want[p, :, o] = c.mass[p, :, o]
    assert torch.equal(want.view(torch.int32), c.mass.view(torch.int32))


@pytest.mark.parametrize("lens,hq,hkv,page", [([1], 1, 1, 16), ([2], 4, 2, 16), ([128], 8, 8, 16), ([129], 8, 1, 32), ([409], 32, 32, 16),
                                              ([5000], 6, 2, 64), ([1, 700, 33, 4097], 32, 8, 16), ([300] * 140, 3, 1, 128),
                                              ([20000], 16, 1, 16), ([777, 1], 128, 1, 16)])
def test_step_adds_the_weights(B, lens, hq, hkv, page):
    run_step(B, lens, hq, hkv, page, want_lse=len(lens) != 2, seed=lens[0], heads_first=page != 32)
    run_step(B, lens, hq, hkv, page, q_scale=5.0, seed=lens[0] + 1)
