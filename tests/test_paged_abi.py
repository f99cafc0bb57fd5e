"""What the entry points of the paged cache refuse, on the host, before anything touches a device."""
import ctypes as C

import pytest

from paper_2406_18139_b200 import binding as B

FAKE = 4096                                     # an aligned address that nothing may follow: these calls must fail first


def paged(hq=8, hkv=2, d=128, page=16, pages=100, stride=10, scale=0.0, **kw):
    lay = B.PagedLayout(hq, hkv, d, page, pages, stride, hkv * page * 128, 128, page * 128, hq * 128, 128, scale)
    for k, v in kw.items():
        setattr(lay, k, v)
    return lay


def ints(*x):
    return (C.c_int * len(x))(*x)


def append(lay=None, layout=None, options=None, cu=(0, 3), lens=(5,), q=FAKE, k=FAKE, v=FAKE, positions=FAKE, q_out=FAKE, cache_k=FAKE,
           cache_v=FAKE, mass=FAKE, table=FAKE, ws=FAKE, ws_bytes=1 << 40):
    layout = layout or B.Layout(8, 2, 128, 8 * 128, 128, 2 * 128, 128, 0.0)
    return B.lib().lookm_append_rows(q, k, v, positions, ints(*cu), ints(*lens), len(lens), C.byref(layout),
                                     None if options is None else C.byref(options), q_out, cache_k, cache_v, mass, table,
                                     C.byref(lay or paged()), ws, ws_bytes, None)


def chunk(lay=None, cu=(0, 3), lens=(5,), q=FAKE, cache_k=FAKE, cache_v=FAKE, table=FAKE, out=FAKE, lse=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return B.lib().lookm_chunk_attention(q, cache_k, cache_v, table, ints(*cu), ints(*lens), len(lens), C.byref(lay or paged()), out, lse, ws,
                                         ws_bytes, None)


def step(lay=None, lens=(5,), q=FAKE, cache_k=FAKE, cache_v=FAKE, mass=FAKE, table=FAKE, out=FAKE, lse=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return B.lib().lookm_step_attention(q, cache_k, cache_v, mass, table, ints(*lens), len(lens), C.byref(lay or paged()), out, lse, ws,
                                        ws_bytes, None)


def evict(lay=None, lens=(5,), budgets=(3,), windows=(1,), cache_k=FAKE, cache_v=FAKE, mass=FAKE, table=FAKE, out_k=FAKE, out_v=FAKE,
          out_mass=FAKE, out_table=FAKE, kept=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return B.lib().lookm_evict(cache_k, cache_v, mass, table, ints(*lens), ints(*budgets), ints(*windows), len(lens), C.byref(lay or paged()),
                               out_k, out_v, out_mass, out_table, kept, ws, ws_bytes, None)


CALLS = [append, chunk, step, evict]


@pytest.mark.parametrize("call", CALLS)
def test_layouts(call):
    bad = dict(hq=0), dict(hkv=0), dict(hq=7), dict(pages=0), dict(stride=0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=3e38), \
        dict(page_stride=0), dict(row_stride=64), dict(head_stride=132), dict(page_stride=-256)
    for kw in bad:
        assert call(paged(**kw)) == B.ERR_INVALID_ARG, kw
    for kw in dict(d=64), dict(page=8), dict(page=24), dict(page=1 << 17), dict(hq=258, hkv=2), dict(page_stride=1 << 40):
        assert call(paged(**kw)) == B.ERR_UNSUPPORTED, kw


@pytest.mark.parametrize("call", CALLS)
def test_lengths_and_pointers(call):
    assert call(lens=(-1,)) == B.ERR_INVALID_ARG
    assert call(lens=(161,)) == B.ERR_INVALID_ARG                  # eleven pages, ten in the table
    assert call(paged(stride=1 << 22), lens=((1 << 25) + 1,)) == B.ERR_UNSUPPORTED
    for name in "cache_k", "cache_v", "table":
        assert call(**{name: None}) == B.ERR_INVALID_ARG
    assert call(cache_k=FAKE + 8) == B.ERR_INVALID_ARG
    assert call(ws=None) == B.ERR_INVALID_ARG
    assert call(ws=FAKE + 128) == B.ERR_INVALID_ARG
    assert call(ws_bytes=0) == B.ERR_WORKSPACE_TOO_SMALL


def test_append_refusals():
    assert append(lens=(158,)) == B.ERR_INVALID_ARG                # the new rows leave the table
    for cu in (1, 3), (0, -1):
        assert append(cu=cu) == B.ERR_INVALID_ARG
    assert append(cu=(0, 5, 3), lens=(1, 1)) == B.ERR_INVALID_ARG
    for kw in dict(k=None), dict(v=None), dict(q=None), dict(q_out=None), dict(q=FAKE + 4), dict(mass=FAKE + 2), dict(q_out=FAKE + 2):
        assert append(**kw) == B.ERR_INVALID_ARG, kw
    for lay in B.Layout(8, 1, 128, 1024, 128, 256, 128, 0.0), B.Layout(4, 2, 128, 512, 128, 256, 128, 0.0), \
            B.Layout(8, 2, 128, 1024, 128, 0, 128, 0.0), B.Layout(8, 2, 128, 1028, 128, 256, 128, 0.0):
        assert append(layout=lay) == B.ERR_INVALID_ARG
    assert append(layout=B.Layout(8, 2, 64, 1024, 128, 256, 128, 0.0)) == B.ERR_UNSUPPORTED
    assert append(paged(q_stride_tok=4)) == B.ERR_INVALID_ARG
    freq = [1.0] * 64
    opt = lambda **kw: B.make_append_options(**{**dict(inv_freq=freq), **kw})
    assert append(options=opt(), positions=None) == B.ERR_INVALID_ARG
    assert append(options=opt(inv_freq=[1.0] * 4)) == B.ERR_UNSUPPORTED            # eight features
    assert append(options=opt(inv_freq=[1.0] * 72)) == B.ERR_INVALID_ARG
    assert append(options=opt(inv_freq=[float("inf")] * 64)) == B.ERR_INVALID_ARG
    o = opt()
    o.inv_freq_host = None
    assert append(options=o) == B.ERR_INVALID_ARG
    for eps in -1.0, float("nan"):
        o = opt(eps=eps)
        o.q_weight = FAKE
        assert append(options=o) == B.ERR_INVALID_ARG
    o = opt()
    o.k_weight = FAKE + 2
    assert append(options=o) == B.ERR_INVALID_ARG


def test_attention_refusals():
    assert chunk(cu=(0, 6)) == B.ERR_INVALID_ARG                   # more new tokens than rows
    assert chunk(cu=(0, 5, 3), lens=(9, 9)) == B.ERR_INVALID_ARG
    assert step(lens=(0,)) == B.ERR_INVALID_ARG
    assert step(mass=None) == B.ERR_INVALID_ARG
    for call in chunk, step:
        for kw in dict(q=None), dict(out=None), dict(q=FAKE + 8), dict(out=FAKE + 4), dict(lse=FAKE + 2):
            assert call(**kw) == B.ERR_INVALID_ARG, kw
        for s in 0, 4, -1024:
            assert call(paged(q_stride_tok=s)) == B.ERR_INVALID_ARG
            assert call(paged(q_stride_head=s)) == B.ERR_INVALID_ARG
    assert B.lib().lookm_chunk_attention(FAKE, FAKE, FAKE, FAKE, None, ints(5), 1, C.byref(paged()), FAKE, FAKE, FAKE, 1 << 40,
                                         None) == B.ERR_INVALID_ARG


def test_evict_refusals():
    for kw in dict(budgets=(0,)), dict(windows=(-1,)), dict(mass=None), dict(out_mass=None), dict(out_k=None), dict(out_table=None), \
            dict(out_v=FAKE + 4), dict(kept=FAKE + 1):
        assert evict(**kw) == B.ERR_INVALID_ARG, kw
    assert evict(kept=None, ws_bytes=256) == B.ERR_WORKSPACE_TOO_SMALL


def test_workspace_sizes_grow_with_what_they_serve():
    size = lambda lens, new=None, **kw: B.lookm_paged_workspace_size(paged(stride=1000, **kw), new, lens)
    assert size([100]) % 256 == 0
    assert 0 < size([100]) <= size([1000]) <= size([1000, 50]) <= size([1000, 900])
    assert size([1000]) <= size([1000], [7]) <= size([1000], [700])
    assert size([]) == size([-1]) == size([16001]) == size([5], [-1]) == size([5], d=64) == 0


@pytest.mark.gpu
def test_binding_refuses_what_the_library_cannot_see():
    import torch
    cpu = torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)
    gpu, q = cpu.cuda(), torch.zeros(1, 2, 128, dtype=torch.bfloat16, device="cuda")
    table = torch.zeros(1, 4, dtype=torch.int32, device="cuda")
    lay = B.make_paged_layout(q, gpu, table)
    ws, out, mass = B.alloc_paged_workspace(lay, None, [5]), torch.empty_like(q), torch.zeros(4, 2, 16, device="cuda")
    ok = lambda **kw: B.lookm_chunk_attention(*[kw.get(n, d) for n, d in dict(q=q, k=gpu, v=gpu, table=table, cu=[0, 1], lens=[5], lay=lay,
                                                                             out=out, lse=None, ws=ws).items()])
    assert ok() == B.OK
    assert ok(k=cpu) == ok(cu=[0, 1, 1]) == ok(table=table.long()) == ok(table=table[:0]) == B.ERR_INVALID_ARG
    assert B.lookm_step_attention(q, gpu, gpu, mass.cpu(), table, [5], lay, out, None, ws) == B.ERR_INVALID_ARG
    assert B.lookm_evict(gpu, gpu, mass, table, [5], [3, 3], [1], lay, gpu, gpu, mass, table, None, ws) == B.ERR_INVALID_ARG
    two, wide = torch.zeros(2, 4, dtype=torch.int32, device="cuda"), torch.zeros(2, 5, dtype=torch.int32, device="cuda")
    assert B.lookm_evict(gpu, gpu, mass, two, [5, 5], [3, 3], [1, 1], lay, gpu, gpu, mass, wide, None, ws) == B.ERR_INVALID_ARG

