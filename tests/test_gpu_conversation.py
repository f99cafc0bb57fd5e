"""The paged cache's operators together, as a conversation uses them, and the ways of calling them: graphs, streams, shared pages, far
pages.  Tolerances: those of the single operators' tests."""
import math

import pytest
import torch

from tests.paged import Cache, D, attention64, kept64
from tests.test_gpu_chunk import close, reference
from tests.test_gpu_paged import freqs, same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2406_18139_b200 import binding
    binding.lib()
    return binding


def test_a_conversation(B):
    """Prompt through the operators, compressed with the log-sum-exp they left straight into a run of pages, a second turn, generated
    tokens with their weights, an eviction, another token."""
    hq, hkv, L, budget, cap, page = 8, 2, 700, 140, 256, 16
    gen = torch.Generator().manual_seed(5)
    normal = lambda *s: torch.randn(*s, generator=gen).cuda()
    qw, kw = ((1 + 0.1 * normal(D)).bfloat16() for _ in range(2))
    opt = B.make_append_options(qw, kw, 1e-6, freqs(128))

    def pool(rows):                               # [hkv, rows, 128], seen as pages of 16 rows
        t = torch.full((hkv, rows, D), math.nan, dtype=torch.bfloat16, device="cuda")
        return t, t.view(hkv, rows // page, page, D).transpose(0, 1)

    def project(n):                               # what a layer's projections leave: one buffer for q, k and v
        return normal(n, hq + 2 * hkv, D).bfloat16().split([hq, hkv, hkv], dim=1)

    table = lambda rows: torch.arange(rows // page, dtype=torch.int32, device="cuda")[None]
    # the prompt: append, attend
    rows = (L + page - 1) // page * page
    (k_all, k_pages), (v_all, v_pages), tab = pool(rows), pool(rows), table(rows)
    q, k, v = project(L)
    qr, pos = torch.empty(L, hq, D, dtype=torch.bfloat16, device="cuda"), torch.arange(L, dtype=torch.int32, device="cuda")
    lay = B.make_paged_layout(qr, k_pages, tab)
    ws = B.alloc_paged_workspace(lay, [L], [L])
    B.check(B.lookm_append_rows(q, k, v, pos, [0, L], [0], B.make_layout(q, k), opt, qr, k_pages, v_pages, None, tab, lay, ws))
    out, lse = torch.empty_like(qr), torch.empty(hq, L, device="cuda")
    B.check(B.lookm_chunk_attention(qr, k_pages, v_pages, tab, [0, L], [L], lay, out, lse, ws))
    B.check(B.lookm_device_status(ws))
    # compression from these rows: with the log-sum-exp as given, and with the library's own sweep
    kp, vp = k_all[:, :L].transpose(0, 1), v_all[:, :L].transpose(0, 1)
    mask = ((pos > 50) & (pos < 627)).to(torch.uint8)
    clay = B.make_layout(qr, kp)
    cws = B.alloc_workspace(clay, [L])
    got = []
    for given in (lse, None):
        (ck_all, ck), (cv_all, cv) = pool(cap), pool(cap)
        o = B.make_options(lse=given, out_stride_head=cap * D)
        st, n = B.lookm_compress_layer_opt(qr, kp, vp, mask, L, budget, 16, B.MERGE_PIVOTAL, clay, o, ck_all, cv_all, cws)
        B.check(st)
        B.check(B.lookm_device_status(cws))
        scores, lists = B.read_intermediates(cws, clay, [L], [budget])
        got.append((ck, cv, torch.from_numpy(scores.copy()), lists))
        assert n == budget
    (ck, cv, scores, lists), other = got[0], got[1]
    assert ((scores - other[2]).abs() <= 1e-4 * other[2].abs()).all()
    # the cache goes on from there; the kept rows' scores are their mass
    c = Cache([0], hkv, page, 1)
    c.k, c.v, c.table, c.lens = ck, cv, table(cap), [budget]
    c.mass = torch.full((cap // page, hkv, page), math.nan, device="cuda")
    p, o = c.where(0, 0, budget)
    for h in range(hkv):
        c.mass[p, h, o] = scores[h][torch.from_numpy(lists[0][h][0].copy()).long()].cuda()
    spare = torch.empty(64, hq, D, dtype=torch.bfloat16, device="cuda")
    lay = B.make_paged_layout(spare, c.k, c.table)
    ws = B.alloc_paged_workspace(lay, [64], [cap])
    seen, rows = L, budget

    def turn(n, with_weights):
        nonlocal seen, rows
        q, k, v = project(n)
        qr = torch.empty(n, hq, D, dtype=torch.bfloat16, device="cuda")
        pos = torch.arange(seen, seen + n, dtype=torch.int32, device="cuda")
        B.check(B.lookm_append_rows(q, k, v, pos, [0, n], [rows], B.make_layout(q, k), opt, qr, c.k, c.v, c.mass, c.table, lay, ws))
        seen, rows = seen + n, rows + n
        c.lens = [rows]
        out, lse, old = torch.empty_like(qr), torch.empty(hq, n, device="cuda"), c.rows(c.mass, 0, rows).double()
        if with_weights:
            B.check(B.lookm_step_attention(qr, c.k, c.v, c.mass, c.table, [rows], lay, out, lse, ws))
        else:
            B.check(B.lookm_chunk_attention(qr, c.k, c.v, c.table, [0, n], [rows], lay, out, lse, ws))
        B.check(B.lookm_device_status(ws))
        ref, ref_lse, w, tol, tol_lse, tol_w = reference(c, 0, qr, n, D ** -0.5)
        assert close(out, ref, tol) and close(lse, ref_lse, tol_lse)
        if with_weights:
            want, room = (x[:, 0].view(hkv, hq // hkv, rows).sum(1).t() for x in (w, tol_w))
            assert ((c.rows(c.mass, 0, rows).double() - old - want).abs() <= room + 2.0 ** -21 * (old + want)).all()

    turn(41, False)
    for _ in range(4):
        turn(1, True)
    keep = 150
    m = c.rows(c.mass, 0, rows).t().cpu().tolist()
    ref = [kept64(m[h], keep, 8) for h in range(hkv)]
    want_k = torch.stack([c.rows(c.k, 0, rows)[torch.tensor(ref[h], device="cuda"), h] for h in range(hkv)], dim=1)
    B.check(B.lookm_evict(c.k, c.v, c.mass, c.table, [rows], [keep], [8], lay, c.k, c.v, c.mass, c.table, None, ws))
    assert same(c.rows(c.k, 0, keep), want_k)
    rows = keep
    turn(1, True)
    turn(3, False)


def step_state(B, seed, lens=(300, 17, 1200), hq=8, hkv=2, page=16):
    c = Cache(lens, hkv, page, seed, room=4)
    n = len(lens)
    c.q = c.normal(n, hq, D).bfloat16()
    c.kn, c.vn = (c.normal(n, hkv, D).bfloat16() for _ in range(2))
    c.pos = torch.tensor(lens, dtype=torch.int32, device="cuda")
    c.qr, c.out, c.lse = torch.empty_like(c.q), torch.empty_like(c.q), torch.empty(hq, n, device="cuda")
    c.paged = B.make_paged_layout(c.qr, c.k, c.table)
    c.ws = B.alloc_paged_workspace(c.paged, None, [x + 1 for x in lens])
    c.opt = B.make_append_options(inv_freq=freqs(64), interleaved=True)
    c.keep = [x * 4 // 5 for x in lens]
    c.kept = torch.empty(hkv * sum(c.keep), dtype=torch.int32, device="cuda")
    return c


def step_calls(B, c):
    n, after = len(c.lens), [x + 1 for x in c.lens]
    B.check(B.lookm_append_rows(c.q, c.kn, c.vn, c.pos, list(range(n + 1)), c.lens, B.make_layout(c.q, c.kn), c.opt, c.qr, c.k, c.v, c.mass,
                                c.table, c.paged, c.ws))
    B.check(B.lookm_step_attention(c.qr, c.k, c.v, c.mass, c.table, after, c.paged, c.out, c.lse, c.ws))
    B.check(B.lookm_chunk_attention(c.qr, c.k, c.v, c.table, list(range(n + 1)), after, c.paged, c.out, c.lse, c.ws))
    B.check(B.lookm_evict(c.k, c.v, c.mass, c.table, after, c.keep, [4] * n, c.paged, c.k, c.v, c.mass, c.table, c.kept, c.ws))


def step_results(c):
    return [x.clone() for x in (c.out, c.lse, c.mass, c.kept, c.k, c.v)]


@pytest.mark.parametrize("lens", [(300, 17, 1200), (9000,)])
def test_captured_and_replayed(B, lens):
    c, d = step_state(B, 3, lens), step_state(B, 3, lens)
    step_calls(B, c)
    step_calls(B, c)
    want = step_results(c)
    warm = step_state(B, 4, lens)                 # function attributes are set before the capture
    step_calls(B, warm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step_calls(B, d)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    B.check(B.lookm_device_status(d.ws))
    assert all(same(a, b) for a, b in zip(want, step_results(d)))


def test_two_streams_with_workspaces_of_their_own(B):
    alone = []
    for seed in (7, 8):
        c = step_state(B, seed, (5000, 900))
        step_calls(B, c)
        alone.append(step_results(c))
    both, streams = [step_state(B, seed, (5000, 900)) for seed in (7, 8)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for c, s in zip(both, streams):
        with torch.cuda.stream(s):
            step_calls(B, c)
    torch.cuda.synchronize()
    for c, want in zip(both, alone):
        B.check(B.lookm_device_status(c.ws))
        assert all(same(a, b) for a, b in zip(want, step_results(c)))


def test_requests_share_the_pages_of_a_prefix(B):
    c = Cache([64 + 20, 64 + 50, 64 + 7], 2, 16, 11)
    for r in (1, 2):                              # the first four pages are request 0's
        c.table[r, :4] = c.table[0, :4]
    q = c.normal(3 * 7, 4, D).bfloat16()
    paged = B.make_paged_layout(q, c.k, c.table)
    ws = B.alloc_paged_workspace(paged, [7] * 3, c.lens)
    out = torch.empty_like(q)
    B.check(B.lookm_chunk_attention(q, c.k, c.v, c.table, [0, 7, 14, 21], c.lens, paged, out, None, ws))
    for r in range(3):
        ref, _, _, tol, _, _ = reference(c, r, q[7 * r:7 * r + 7], 7, D ** -0.5)
        assert close(out[7 * r:7 * r + 7], ref, tol)


def test_evict_to_other_pages_of_the_same_pool(B):
    c = Cache([500], 3, 16, 12, spare=40)
    used = set(c.table[0].tolist())
    free = [x for x in range(len(c.k)) if x not in used]
    table = torch.tensor([free[:c.table.shape[1]]], dtype=torch.int32, device="cuda")
    old = c.k.clone(), c.v.clone(), c.mass.clone()
    m = c.rows(c.mass, 0, 500).t().cpu().tolist()
    paged = B.make_paged_layout(None, c.k, c.table, n_q_heads=3)
    ws = B.alloc_paged_workspace(paged, None, [500])
    B.check(B.lookm_evict(c.k, c.v, c.mass, c.table, [500], [333], [5], paged, c.k, c.v, c.mass, table, None, ws))
    p, o = c.where(0, 0, 333, table)
    for h in range(3):
        idx = torch.tensor(kept64(m[h], 333, 5), device="cuda")
        src, so = c.table[0].long()[idx // 16], idx % 16
        for a, b in zip(old, (c.k, c.v, c.mass)):
            want = a[src, h, so]
            assert same(b[p, h, o], want)
            a[p, h, o] = want
    assert all(same(a, b) for a, b in zip(old, (c.k, c.v, c.mass)))


def test_pages_beyond_32_bit_offsets(B):
    """Pools of 4.8 GB each whose used pages lie at both ends: offsets beyond 2^31 elements and 2^32 bytes."""
    hkv, page, lens = 8, 64, [200]
    pages = (5 << 30) // (2 * hkv * page * D) * 15 // 16
    c = Cache(lens, hkv, page, 13)
    small = c.k, c.v
    big = [torch.empty(pages, hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    assert big[0].numel() > 1 << 31
    mass = torch.zeros(pages, hkv, page, device="cuda")
    to = torch.tensor([[pages - 1, 0, pages - 2, 1]], dtype=torch.int32, device="cuda")
    for b, s in zip(big, small):
        b[to[0].long()] = s[c.table[0].long()]
    q, kn, vn = (c.normal(2, h, D).bfloat16() for h in (16, hkv, hkv))
    out, want, before = torch.empty_like(q), torch.empty_like(q), c.mass.clone()
    for k, v, table, o, m in ((small[0], small[1], c.table, want, c.mass), (big[0], big[1], to, out, mass)):
        paged = B.make_paged_layout(q, k, table)
        ws = B.alloc_paged_workspace(paged, [2], [202])
        B.check(B.lookm_append_rows(q, kn, vn, None, [0, 2], [198], B.make_layout(q, kn), None, o, k, v, m, table, paged, ws))
        B.check(B.lookm_chunk_attention(q, k, v, table, [0, 2], [200], paged, o, None, ws))
        B.check(B.lookm_step_attention(q[:1], k, v, m, table, [200], paged, o[:1], None, ws))
        m[table[0].long()] = before[c.table[0].long()]             # (the same masses for both evictions)
        B.check(B.lookm_evict(k, v, m, table, [200], [120], [3], paged, k, v, m, table, None, ws))
        B.check(B.lookm_device_status(ws))
    assert same(out, want)
    for b, s in zip(big, small):
        assert same(b[to[0].long()][:, :, :], s[c.table[0].long()])
