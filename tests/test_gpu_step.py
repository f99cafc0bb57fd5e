"""Steps with weights over a paged cache, through the C ABI, against fp64: what a row's mass receives.  Tolerances: those of the single
operators' tests, and for each of the k additions to a mass half a step of it (2^-24 of the sum)."""
import math

import pytest
import torch

from tests.paged import Cache, D
from tests.test_gpu_chunk import close, reference
from tests.test_gpu_paged import same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2406_18139_b200 import binding
    binding.lib()
    return binding


def step(B, c, q, hq, lse=None, scale=0.0, lens=None):
    lens = c.lens if lens is None else lens
    out = torch.empty(len(lens), hq, D, dtype=torch.bfloat16, device="cuda")
    paged = B.make_paged_layout(q, c.k, c.table, scale)
    ws = B.alloc_paged_workspace(paged, None, lens)
    ws[256:] = 255
    B.check(B.lookm_step_attention(q, c.k, c.v, c.mass, c.table, lens, paged, out, lse, ws))
    B.check(B.lookm_device_status(ws))
    return out


@pytest.mark.parametrize("prefix,tails,hq,hkv,page", [
    (64, [20, 50, 7], 4, 2, 16),                                       # short caches: weights in the first launch
    (512, [1, 1, 100, 300, 17, 64, 2, 90], 8, 8, 32),
    (4096, [30, 1000, 1], 8, 2, 64),                                   # long ones: in the second; units cut
    (2048, [i % 50 + 1 for i in range(140)], 2, 1, 128)])              # two batches of a call
def test_requests_that_share_a_prefix_add_up_their_weights(B, prefix, tails, hq, hkv, page):
    lens = [prefix + t for t in tails]
    c = Cache(lens, hkv, page, prefix)
    c.table[1:, :prefix // page] = c.table[0, :prefix // page]
    q = c.normal(len(lens), hq, D).bfloat16()
    old = c.mass.clone()
    want, tol, n = old.double().nan_to_num(0), torch.zeros_like(old, dtype=torch.float64), torch.zeros_like(old)
    out = step(B, c, q, hq)
    g = hq // hkv
    for r, k in enumerate(lens):
        ref, _, w, tol_out, _, tol_w = reference(c, r, q[r:r + 1], 1, D ** -0.5)
        assert close(out[r:r + 1], ref, tol_out)
        p, o = c.where(r, 0, k)
        for total, x in ((want, w), (tol, tol_w)):
            total[p, :, o] += x[:, 0].view(hkv, g, k).sum(1).t()
        n[p, :, o] += g + 1
    some = n > 0
    assert ((c.mass.double() - want).abs() <= tol + 2.0 ** -24 * n * want)[some].all()
    assert same(c.mass[~some], old[~some])


def test_rows_that_nobody_shares_do_not_depend_on_timing(B):
    results = []
    for _ in range(3):
        c = Cache([64 + 500, 64 + 3000, 64 + 7], 2, 16, 5)
        c.table[1:, :4] = c.table[0, :4]
        step(B, c, c.normal(3, 8, D).bfloat16(), 8)
        c.mass[c.table[0, :4].long()] = 0
        results.append(c.mass)
    assert same(results[0], results[1]) and same(results[0], results[2])


def test_a_page_that_a_request_names_twice(B):
    """Its rows are seen twice, and both weights reach their mass."""
    c = Cache([48], 1, 16, 6)
    c.table[0, 2] = c.table[0, 0]
    q = c.normal(1, 2, D).bfloat16()
    old = c.mass.clone()
    step(B, c, q, 2)
    _, _, w, _, _, tol_w = reference(c, 0, q, 1, D ** -0.5)
    w, tol_w = (x[:, 0].sum(0) for x in (w, tol_w))
    got = c.mass[c.table[0, 0], 0].double() - old[c.table[0, 0], 0].double()
    assert ((got - w[:16] - w[32:48]).abs() <= tol_w[:16] + tol_w[32:48] + 2.0 ** -24 * 6 * c.mass[c.table[0, 0], 0].abs()).all()


def check(B, c, q, hq, hkv, out, lse, old, scale):
    """Outputs, log-sum-exps and masses of a step, against fp64."""
    for r, k in enumerate(c.lens):
        ref, ref_lse, w, tol, tol_lse, tol_w = reference(c, r, q[r:r + 1], 1, scale)
        assert close(out[r:r + 1], ref, tol), r
        assert close(lse[:, r:r + 1], ref_lse, tol_lse), r
        p, o = c.where(r, 0, k)
        sums, tols = (x[:, 0].view(hkv, hq // hkv, k).sum(1).t() for x in (w, tol_w))
        ref_m = old[p, :, o].double() + sums
        assert close(c.mass[p, :, o], ref_m, tols + 2.0 ** -23 * (hq // hkv + 1) * ref_m.abs()), r


@pytest.mark.parametrize("scale", [0.02, 0.3])
@pytest.mark.parametrize("lens,hq,hkv,page", [([5, 700], 8, 2, 16), ([9000], 4, 4, 64), ([70000], 2, 1, 65536)])
def test_scales(B, scale, lens, hq, hkv, page):
    c = Cache(lens, hkv, page, sum(lens))
    q, lse, old = c.normal(len(lens), hq, D).bfloat16(), torch.empty(hq, len(lens), device="cuda"), c.mass.clone()
    out = step(B, c, q, hq, lse, scale)
    check(B, c, q, hq, hkv, out, lse, old, scale)


@pytest.mark.parametrize("n,hq,hkv,page", [(129, 4, 4, 16), (1500, 8, 2, 16), (9000, 8, 2, 16), (4000, 2, 1, 64)])
@pytest.mark.parametrize("kind", ["v nan", "v inf", "k nan", "k -inf", "k all -inf"])
def test_infinities_and_nan(B, n, hq, hkv, page, kind):
    """What a row holds reaches the outputs and the masses of its head, and no other head's."""
    c = Cache([n], hkv, page, n)
    q = c.normal(1, hq, D).bfloat16()
    k, v = c.rows(c.k, 0, n).float(), c.rows(c.v, 0, n).float()
    if kind == "v nan":
        v[n - 1, 0, 5] = math.nan
    elif kind == "v inf":
        v[n - 1, -1, 0], v[0, 0, 77], v[n // 2, 0, 77], v[n // 2, 0, 3] = math.inf, -math.inf, math.inf, math.inf
    elif kind == "k nan":
        k[n // 2, 0, 9] = math.nan
    else:
        q[..., 4] = 1.0
        k[(slice(None) if "all" in kind else n // 3), 0, 4] = -math.inf
    c.put(c.k, 0, 0, k)
    c.put(c.v, 0, 0, v)
    lse, old = torch.empty(hq, 1, device="cuda"), c.mass.clone()
    out = step(B, c, q, hq, lse)
    check(B, c, q, hq, hkv, out, lse, old, D ** -0.5)


@pytest.mark.parametrize("lens", [[9000 + 400 * (i % 9) for i in range(140)], [300 + i for i in range(300)]])
def test_more_requests_than_a_launch_takes(B, lens):
    c = Cache(lens, 1, 32, 21)
    q, lse, old = c.normal(len(lens), 2, D).bfloat16(), torch.empty(2, len(lens), device="cuda"), c.mass.clone()
    out = step(B, c, q, 2, lse)
    check(B, c, q, 2, 1, out, lse, old, D ** -0.5)
