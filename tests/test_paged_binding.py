"""What the binding of the paged cache refuses because the library, which gets pointers, can't see it.  On the CPU: the library is one that does
nothing but say that it was called, and tensors on the CPU stand for those on the device."""
import pytest
import torch

from paper_2406_18139_b200 import binding as B

HQ, HKV, PAGE, PAGES, NEW, LENS = 4, 2, 16, 9, [3, 2], [20, 33]
bf16 = torch.bfloat16


class Library:
    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*args):
            self.calls += 1
            return B.OK
        return call


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(B, "_lib", lib)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    return lib


def pool():
    return torch.zeros(PAGES, HKV, PAGE, 128, dtype=bf16)


def masses():
    return torch.zeros(PAGES, HKV, PAGE)


def table():
    return torch.zeros(2, 4, dtype=torch.int32)


def rows(heads, n=sum(NEW)):
    return torch.zeros(n, heads, 128, dtype=bf16)


def arguments(call):
    """Names and values of a call that is taken."""
    a = dict(cache_k=pool(), cache_v=pool(), page_table=table(), workspace=torch.zeros(1, dtype=torch.uint8))
    if call == "append":
        a.update(q=rows(HQ), k=rows(HKV), v=rows(HKV), positions=torch.zeros(sum(NEW), dtype=torch.int32), cu=[0, 3, 5], lens=LENS, options=None,
                 q_out=rows(HQ), mass=masses())
        a["layout"] = B.make_layout(a["q"], a["k"])
    elif call == "chunk":
        a.update(q=rows(HQ), cu=[0, 3, 5], lens=LENS, out=rows(HQ), lse=torch.zeros(HQ, sum(NEW)))
    elif call == "step":
        a.update(q=rows(HQ, 2), mass=masses(), lens=LENS, out=rows(HQ, 2), lse=torch.zeros(HQ, 2))
    else:
        a.update(mass=masses(), lens=LENS, budgets=[10, 20], windows=[1, 1], out_k=pool(), out_v=pool(), out_mass=masses(),
                 out_page_table=table(), kept_idx=torch.zeros(HKV * 30, dtype=torch.int32))
    a["paged"] = B.make_paged_layout(a.get("q"), a["cache_k"], a["page_table"], n_q_heads=HQ)
    return a


def run(call, a):
    g = a.__getitem__
    if call == "append":
        names = "q k v positions cu lens layout options q_out cache_k cache_v mass page_table paged workspace"
        return B.lookm_append_rows(*map(g, names.split()))
    if call == "chunk":
        return B.lookm_chunk_attention(*map(g, "q cache_k cache_v page_table cu lens paged out lse workspace".split()))
    if call == "step":
        return B.lookm_step_attention(*map(g, "q cache_k cache_v mass page_table lens paged out lse workspace".split()))
    names = "cache_k cache_v mass page_table lens budgets windows paged out_k out_v out_mass out_page_table kept_idx workspace"
    return B.lookm_evict(*map(g, names.split()))


CALLS = ["append", "chunk", "step", "evict"]


def refused(library, call, **changed):
    a = {**arguments(call), **changed}
    before = library.calls
    assert run(call, a) == B.ERR_INVALID_ARG, changed.keys()
    assert library.calls == before


def taken(library, call, **changed):
    before = library.calls
    assert run(call, {**arguments(call), **changed}) == B.OK and library.calls == before + 1


@pytest.mark.parametrize("call", CALLS)
def test_calls_that_are_taken(library, call):
    taken(library, call)
    for name in {"append": ["mass", "positions"], "chunk": ["lse"], "step": ["lse"], "evict": ["kept_idx"]}[call]:
        taken(library, call, **{name: None})
    if call == "append":
        taken(library, call, q=None, q_out=None)


@pytest.mark.parametrize("call", CALLS)
def test_types(library, call):
    """Positions as torch.arange makes them would be read as pairs of 32-bit numbers, every other one zero; others likewise."""
    a = arguments(call)
    for name, t in a.items():
        if isinstance(t, torch.Tensor) and name != "workspace":
            for other in {torch.int32: (torch.int64, torch.float32), bf16: (torch.float16, torch.float32),
                          torch.float32: (torch.float64, bf16)}[t.dtype]:
                refused(library, call, **{name: t.to(other)})


@pytest.mark.parametrize("call,names", [("append", ["positions", "mass"]), ("chunk", ["out", "lse"]), ("step", ["out", "lse", "mass"]),
                                        ("evict", ["mass", "out_mass", "kept_idx"])])
def test_what_has_to_lie_in_a_row_does_and_is_long_enough(library, call, names):
    a = arguments(call)
    for name in names:
        t = a[name]
        refused(library, call, **{name: t[:-1]})
        refused(library, call, **{name: torch.stack([t, t], dim=-1)[..., 0]})


def test_weights_of_the_norm():
    good = torch.ones(128, dtype=bf16)
    for bad in good, good.float(), good[:64]:                # (the first lies on the CPU, and the library would follow its address)
        with pytest.raises(AssertionError):
            B.make_append_options(bad, None, 1e-6)
        with pytest.raises(AssertionError):
            B.make_append_options(None, bad, 1e-6)


@pytest.mark.parametrize("call", CALLS)
def test_tables_that_are_not_the_layouts(library, call):
    """The library goes by the layout's stride: entries of other requests, or what lies behind the table, would be taken for page numbers."""
    names = ["page_table"] + (["out_page_table"] if call == "evict" else [])
    wide, one = torch.zeros(2, 6, dtype=torch.int32), dict(lens=LENS[1:], **{"append": dict(cu=[0, 5]), "chunk": dict(cu=[0, 5]), "step": {},
                                                                             "evict": dict(budgets=[30], windows=[1])}[call])
    last = LENS[1] + (5 if call == "append" else 0)          # rows of a single request's cache: three pages
    assert 2 * PAGE < last <= 3 * PAGE
    for name in names:
        refused(library, call, **{name: wide})               # it has grown since the layout was made
        refused(library, call, **{name: wide[:, :4].contiguous()[:1]})
        refused(library, call, **{name: torch.zeros(4, 2, dtype=torch.int32).t()})
        refused(library, call, **{name: torch.zeros(8, dtype=torch.int32)})
        refused(library, call, **{name: None})
        refused(library, call, **{name: table()[:, :2] if name == "page_table" else table()[:, :1]})
        taken(library, call, **{name: wide[:1]}, **one)      # one request: no other row is looked for
        taken(library, call, **{name: torch.zeros(1, 3, dtype=torch.int32)}, **one)          # fewer columns, and enough
        refused(library, call, **{name: torch.zeros(1, 2 if name == "page_table" else 1, dtype=torch.int32)}, **one)
    both = torch.zeros(2, 10, dtype=torch.int32)[:, :4]      # (a stride that is not the number of columns)
    a = arguments(call)
    taken(library, call, **{name: both for name in names}, paged=B.make_paged_layout(a.get("q"), a["cache_k"], both, n_q_heads=HQ))


def apart(t):
    """The same numbers with a gap behind every first index."""
    wide = torch.zeros(t.shape[0], 2, *t.shape[1:], dtype=t.dtype)
    wide[:, 0] = t
    return wide[:, 0]


POOLS = {"append": ["cache_k", "cache_v"], "chunk": ["cache_k", "cache_v"], "step": ["cache_k", "cache_v"],
         "evict": ["cache_k", "cache_v", "out_k", "out_v"]}


@pytest.mark.parametrize("call", CALLS)
def test_pools_that_are_not_the_layouts(library, call):
    """One layout stands for all pools of a call: another pool's strides would be taken for its own."""
    more = torch.zeros(PAGES + 2, HKV, PAGE, 128, dtype=bf16)
    for name in POOLS[call]:
        refused(library, call, **{name: torch.zeros(PAGES, PAGE, HKV, 128, dtype=bf16).transpose(1, 2)})
        refused(library, call, **{name: apart(pool())})
        refused(library, call, **{name: pool()[:-1]})
        refused(library, call, **{name: torch.zeros(PAGES, 2 * HKV, PAGE, 128, dtype=bf16)[:, :HKV]})
        refused(library, call, **{name: torch.zeros(PAGES, HKV, 128, PAGE, dtype=bf16).transpose(2, 3)})
        refused(library, call, **{name: None})
        taken(library, call, **{name: more})                 # further pages that no table names
    rows_first = {name: torch.zeros(PAGES, PAGE, HKV, 128, dtype=bf16).transpose(1, 2) for name in POOLS[call]}
    a = arguments(call)
    taken(library, call, **rows_first, paged=B.make_paged_layout(a.get("q"), rows_first["cache_k"], a["page_table"], n_q_heads=HQ))
    # a dimension of one may have any stride
    one = {name: torch.zeros(PAGES, 3, PAGE, 128, dtype=bf16)[:, :1] for name in POOLS[call]}
    same = {name: torch.zeros(PAGES, 1, PAGE, 128, dtype=bf16).expand(PAGES, 1, PAGE, 128) for name in POOLS[call]}
    if call in ("chunk", "step"):
        taken(library, call, **one, paged=B.make_paged_layout(a["q"], one["cache_k"], a["page_table"]))
        refused(library, call, **same, paged=B.make_paged_layout(a["q"], one["cache_k"], a["page_table"]))


@pytest.mark.parametrize("call,names", [("append", ["q", "k", "v", "q_out"]), ("chunk", ["q"]), ("step", ["q"])])
def test_rows_of_new_tokens_that_are_not_the_layouts(library, call, names):
    a = arguments(call)
    for name in names:
        t = a[name]
        refused(library, call, **{name: apart(t)})
        refused(library, call, **{name: t[:-1]})
        refused(library, call, **{name: torch.cat([t, t], dim=1)})
        refused(library, call, **{name: torch.cat([t, t], dim=1)[:, ::2]})
        refused(library, call, **{name: t.reshape(len(t), -1)})
        taken(library, call, **{name: torch.cat([t, t])})
        if name in ("k", "v"):
            refused(library, call, **{name: None})
    if call == "append":                                     # one buffer of q, k and v, as a fused projection leaves it
        q, k, v = rows(HQ + 2 * HKV).split([HQ, HKV, HKV], dim=1)
        taken(library, call, q=q, k=k, v=v, layout=B.make_layout(q, k))
        refused(library, call, q=q, k=k, layout=B.make_layout(q, k))                       # (v lies otherwise)


def test_a_single_token_may_have_any_stride(library):
    a = arguments("append")
    q, k, v = rows(HQ + 2 * HKV, 1).split([HQ, HKV, HKV], dim=1)
    taken(library, "append", q=q, k=k, v=rows(HKV, 1), q_out=rows(HQ, 7)[:1], cu=[0, 1, 1], layout=B.make_layout(q, k))
    taken(library, "chunk", q=rows(2 * HQ, 1)[:, :HQ], cu=[0, 1, 1])
    taken(library, "chunk", q=a["q"][:0], cu=[0, 0, 0])
