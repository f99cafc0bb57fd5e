"""The operators of a conversation that goes on over a paged cache, as cases that can be timed and compared.

Four operators, each through the binding of the C ABI (`own`) and in a plain form of elementary torch operations:

  append  new tokens' queries and keys normed per head and rotated to their positions, keys and values
          written to the cache's pages (lookm_append_rows)
  chunk   attention of each request's newest tokens over its paged cache, causal among themselves, with the
          rows' log-sum-exp (lookm_chunk_attention): a prompt, a later turn of a conversation, single tokens
  step    attention of one new token per request that also adds every cached row's weight to the row's
          accumulated mass (lookm_step_attention)
  evict   the rows of least accumulated mass leave the cache, the recent ones and the heaviest of the others
          stay, in their order (lookm_evict)

A cache is a pool of pages, seen as [pages, KV heads, rows of a page, 128] whatever its strides, and a table
of page numbers per request; row t of request r is row t % rows of page table[r, t // rows].  `mass` is fp32
[pages, KV heads, rows of a page].

Head counts, cache lengths, budgets and windows are those of the package's workloads and of the ranges
between and around them.  Queries and values are N(0, 1); keys are N(0, 1) with four sinks and some salient
rows that draw attention, as in prompts.  Pages lie scattered over the pool, and what no request owns holds
other requests' old rows.
"""
import math
import random

import torch

own = False

D = 128                                            # head_dim, the only one the library has
HEADS = ((8, 8), (32, 32), (40, 40), (32, 8))      # (query heads, KV heads)
PAGES = (16, 32, 64, 128)                          # rows of a page
THETA = 10000.0
EPS = 1e-6
SALIENT_LOGIT = 5.0
MOST_PAIRS = 8192 * 8192 // 2 * 32                 # (query, key) pairs of the largest prompt, over its heads
MOST_ROWS = 1 << 20                                # cached rows over all requests and KV heads


def listed():
    return [
        # One generated token of one request: the smallest call there is, all latency.
        append("append_1_32h_8kv", 1, 1, 1, 32, 8, 16),
        # A short prompt with one image, rotated but not normed (a model without such norms).
        append("append_700_32h", 1, 700, 700, 32, 32, 16, norm=False),
        # A serving batch's prefill: 16 ragged prompts, half of the features rotated in adjacent pairs.
        append("append_16_ragged_40h", 16, 64, 2048, 40, 40, 64, rotary=64, interleaved=True),
        # Sixteen conversations generate a token each over ragged caches.
        chunk("chunk_16_single_32h_8kv", 16, 1, 1, 400, 8192, 32, 8, 16),
        # The short prompt itself: nothing lies before it.
        chunk("chunk_700_prompt_32h", 1, 700, 700, 0, 0, 32, 32, 16),
        # The 8192-token prompt of 32 heads, the headline shape.  The largest.
        chunk("chunk_8192_prompt_32h", 1, 8192, 8192, 0, 0, 32, 32, 128),
        # A later turn: 512 new tokens over a long conversation, grouped queries.
        chunk("chunk_512_over_32768_32h_8kv", 1, 512, 512, 32256, 32256, 32, 8, 64),
        # Sixteen users' next questions, of 1 to 200 tokens, over caches of 400 to 16384 rows.
        chunk("chunk_16_ragged_32h_8kv", 16, 1, 200, 400, 16384, 32, 8, 32),
        # A generated token over a cache at 5 % of an 8192-token prompt, weights accumulated.
        step("step_409_32h", 1, 409, 409, 32, 32, 16),
        # ... for sixteen requests over ragged, long caches.
        step("step_16_ragged_32h_8kv", 16, 400, 16384, 32, 8, 64),
        # An 8192-row cache brought down to 20 %, to pages of its own (the old ones are shared).
        evict("evict_8192_32h_8kv", 1, 8192, 8192, 32, 8, 16, 0.2),
        # Sixteen caches that outgrew their budget by a quarter, in place.
        evict("evict_16_ragged_32h", 16, 1000, 8192, 32, 32, 64, 0.8, in_place=True),
    ]


def append(name, n, fewest, most, hq, hkv, page, norm=True, rotary=128, interleaved=False, heads_first=True, lengths=0):
    return {"name": name, "kind": "append", "n": n, "fewest": fewest, "most": most, "shortest": 0, "longest": 1000, "hq": hq,
            "hkv": hkv, "page": page, "norm": norm, "rotary": rotary, "interleaved": interleaved, "heads_first": heads_first,
            "lengths": lengths}


def chunk(name, n, fewest, most, shortest, longest, hq, hkv, page, heads_first=True, lengths=0):
    """`fewest` to `most` new tokens per request over `shortest` to `longest` rows that lie before them."""
    return {"name": name, "kind": "chunk", "n": n, "fewest": fewest, "most": most, "shortest": shortest, "longest": longest,
            "hq": hq, "hkv": hkv, "page": page, "heads_first": heads_first, "lengths": lengths}


def step(name, n, shortest, longest, hq, hkv, page, heads_first=True, lengths=0):
    return {"name": name, "kind": "step", "n": n, "fewest": 1, "most": 1, "shortest": shortest, "longest": longest, "hq": hq,
            "hkv": hkv, "page": page, "heads_first": heads_first, "lengths": lengths}


def evict(name, n, shortest, longest, hq, hkv, page, ratio, window=32, in_place=False, heads_first=True, lengths=0):
    return {"name": name, "kind": "evict", "n": n, "fewest": 0, "most": 0, "shortest": shortest, "longest": longest, "hq": hq,
            "hkv": hkv, "page": page, "ratio": ratio, "window": window, "in_place": in_place, "heads_first": heads_first,
            "lengths": lengths}


def draw(rng):
    """Sizes over the whole range of their kind, by logarithm; odd ones are the rule."""
    def between(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    kind = rng.choice(["append", "chunk", "chunk", "chunk", "step", "evict"])
    hq, hkv = rng.choice(HEADS)
    page, heads_first, lengths = rng.choice(PAGES), rng.random() < 0.7, rng.randrange(1 << 20)
    n = rng.choice([1, 1, rng.randint(2, 16)])
    rows = MOST_ROWS // (n * hkv)
    if kind == "append":
        lo = between(1, 500)
        case = append("", n, lo, between(lo, 2048), hq, hkv, page, rng.random() < 0.6, rng.choice([128, 128, 64, 32]),
                      rng.random() < 0.4, heads_first, lengths)
    elif kind == "chunk":
        use = rng.choice(["single", "prompt", "turn"])
        if use == "single":
            lo = between(100, min(32768, rows))
            case = chunk("", n, 1, 1, lo, between(lo, min(32768, rows)), hq, hkv, page, heads_first, lengths)
        elif use == "prompt":
            longest = int(math.sqrt(2 * MOST_PAIRS / (hq * n)))
            hi = between(100, min(8192, longest))
            case = chunk("", n, between(50, hi), hi, 0, 0, hq, hkv, page, heads_first, lengths)
        else:
            lo = between(100, min(32000, rows))
            hi = between(lo, min(32000, rows))
            most = between(2, max(2, min(1024, MOST_PAIRS // (n * hq * (hi + 1024)))))
            case = chunk("", n, between(1, most), most, lo, hi, hq, hkv, page, heads_first, lengths)
    elif kind == "step":
        lo = between(100, min(32768, rows))
        case = step("", n, lo, between(lo, min(32768, rows)), hq, hkv, page, heads_first, lengths)
    else:
        hi = between(640, min(32768, rows))
        case = evict("", n, between(300, hi), hi, hq, hkv, page, rng.choice([0.05, 0.2, 0.5, 0.8, 0.95]),
                     rng.choice([1, 16, 32, 64]), rng.random() < 0.5, heads_first, lengths)
    del case["name"]
    return case


def sizes_of(case):
    """(new tokens, cached rows with these included) per request, fixed by the case alone."""
    rng = random.Random(case["lengths"])
    new = [rng.randint(case["fewest"], case["most"]) for _ in range(case["n"])]
    old = [rng.randint(case["shortest"], case["longest"]) for _ in range(case["n"])]
    return new, [a + b for a, b in zip(new, old)]


def budgets_of(case, lens):
    return [max(1, int(case["ratio"] * n)) for n in lens]


# ---- inputs -------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    hq, hkv, page = case["hq"], case["hkv"], case["page"]
    new, lens = sizes_of(case)
    n, total = case["n"], sum(new)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def pool(pages):
        if case["heads_first"]:
            return normal(pages, hkv, page, D).bfloat16()
        return normal(pages, page, hkv, D).bfloat16().transpose(1, 2)

    most = max(-(-x // page) for x in lens)
    pages = sum(-(-x // page) for x in lens) + 3
    s = {"case": case, "new": new, "lens": lens, "cu": [sum(new[:i]) for i in range(n + 1)]}
    s["cache_k"], s["cache_v"] = pool(pages), pool(pages)
    s["table"], at = torch.zeros(n, most, dtype=torch.int32), 0
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).int()
    for r, x in enumerate(lens):
        k = -(-x // page)
        s["table"][r, :k] = order[at:at + k]
        at += k
    s["table"] = s["table"].cuda()
    # (request, row) of every new token and of every cached row, for the plain forms
    s["new_at"] = index_of([(r, lens[r] - new[r], new[r]) for r in range(n)])
    s["row_at"] = index_of([(r, 0, lens[r]) for r in range(n)])
    s["mass"] = torch.exp(2.0 * normal(pages, hkv, page))
    if case["kind"] == "append":
        s["q"], s["k"], s["v"] = (normal(total, h, D).bfloat16() * 2 for h in (hq, hkv, hkv))
        s["positions"] = (s["new_at"][1] + 37).int()
        s["q_out"] = torch.empty_like(s["q"])
        s["q_weight"], s["k_weight"] = ((1 + 0.2 * normal(D)).bfloat16() if case["norm"] else None for _ in range(2))
        s["inv_freq"] = [THETA ** (-2.0 * i / case["rotary"]) for i in range(case["rotary"] // 2)]
    elif case["kind"] == "evict":
        s["budgets"], s["windows"] = budgets_of(case, lens), [case["window"]] * n
        s["budget"], s["window"], s["len"] = (torch.tensor(x, device="cuda") for x in (s["budgets"], s["windows"], lens))
        s["kept"] = torch.zeros(hkv * sum(s["budgets"]), dtype=torch.int32, device="cuda")
        s["out_mass"] = torch.zeros_like(s["mass"])
        if case["in_place"]:
            s["out_k"], s["out_v"], s["out_table"] = s["cache_k"], s["cache_v"], s["table"]
        else:
            s["out_k"], s["out_v"], s["out_table"] = s["cache_k"].clone(), s["cache_v"].clone(), pages - 1 - s["table"]
    else:
        salient(s, normal, hq, hkv, total)
        s["out"] = torch.empty(total, hq, D, dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty(hq, total, device="cuda")
    return s


def index_of(spans):
    """Request and row number of spans (request, first row, rows), one after another."""
    at = [torch.cat([x.new_empty(0) if not len(x) else x for x in parts]) for parts in
          zip(*[(torch.full((k,), r), torch.arange(a, a + k)) for r, a, k in spans])]
    return [x.cuda() for x in at]


def salient(s, normal, hq, hkv, total):
    """Queries, and rows of the caches that draw attention: the first four of a request and one in fifty."""
    page = s["case"]["page"]
    u = torch.nn.functional.normalize(normal(hkv, D), dim=-1)
    s["q"] = (normal(total, hq, D) + 5.0 * u.repeat_interleave(hq // hkv, dim=0)).bfloat16()
    r, t = s["row_at"]
    at = s["table"][r, t // page].long(), t % page
    hit = (t < 4) | (normal(len(t)) > 2.05)
    k = s["cache_k"][at[0], :, at[1]].float()
    k -= (k * u).sum(-1, keepdim=True) * u
    k += (SALIENT_LOGIT * math.sqrt(D) / 5.0) * hit[:, None, None] * u
    s["cache_k"][at[0], :, at[1]] = k.bfloat16()


# ---- the pass -----------------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if own:
        run_own(s, kind)
    elif kind == "append":
        plain_append(s)
    elif kind == "evict":
        plain_evict(s)
    else:
        plain_attention(s, kind == "step")
    if kind == "append":
        return {"q": s["q_out"], "cache_k": s["cache_k"], "cache_v": s["cache_v"], "mass": s["mass"]}
    if kind == "evict":
        return {"out_k": s["out_k"], "out_v": s["out_v"], "out_mass": s["out_mass"], "kept": s["kept"]}
    return {"out": s["out"], "lse": s["lse"], **({"mass": s["mass"]} if kind == "step" else {})}


def run_own(s, kind):
    from paper_2406_18139_b200 import binding as B

    if "workspace" not in s:                       # what a server sets up once per cache
        q = s.get("q") if kind != "evict" else None
        s["paged"] = B.make_paged_layout(q, s["cache_k"], s["table"], n_q_heads=s["case"]["hq"])
        s["workspace"] = B.alloc_paged_workspace(s["paged"], s["new"], s["lens"])
        if kind == "append":
            s["layout"] = B.make_layout(s["q"], s["k"])
            s["options"] = B.make_append_options(s["q_weight"], s["k_weight"], EPS, s["inv_freq"], s["case"]["interleaved"])
    if kind == "append":
        before = [a - b for a, b in zip(s["lens"], s["new"])]
        status = B.lookm_append_rows(s["q"], s["k"], s["v"], s["positions"], s["cu"], before, s["layout"], s["options"], s["q_out"],
                                     s["cache_k"], s["cache_v"], s["mass"], s["table"], s["paged"], s["workspace"])
    elif kind == "chunk":
        status = B.lookm_chunk_attention(s["q"], s["cache_k"], s["cache_v"], s["table"], s["cu"], s["lens"], s["paged"], s["out"],
                                         s["lse"], s["workspace"])
    elif kind == "step":
        status = B.lookm_step_attention(s["q"], s["cache_k"], s["cache_v"], s["mass"], s["table"], s["lens"], s["paged"], s["out"],
                                        s["lse"], s["workspace"])
    else:
        status = B.lookm_evict(s["cache_k"], s["cache_v"], s["mass"], s["table"], s["lens"], s["budgets"], s["windows"], s["paged"],
                               s["out_k"], s["out_v"], s["out_mass"], s["out_table"], s["kept"], s["workspace"])
    B.check(status)


def plain_append(s):
    """y = x / sqrt(mean(x^2) + eps) * w per head; pairs of features turned by position * frequency."""
    case, page = s["case"], s["case"]["page"]
    angle = s["positions"].double()[:, None] * torch.tensor(s["inv_freq"], dtype=torch.float64, device="cuda")
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    r, t = s["new_at"]
    at, row = s["table"][r, t // page].long(), t % page
    s["q_out"].copy_(norm_rotate(s["q"], s["q_weight"], cos, sin, case))
    s["cache_k"][at, :, row] = norm_rotate(s["k"], s["k_weight"], cos, sin, case).bfloat16()
    s["cache_v"][at, :, row] = s["v"]
    s["mass"][at, :, row] = 0.0


def norm_rotate(x, weight, cos, sin, case):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
    turned, rest = x[..., :case["rotary"]], x[..., case["rotary"]:]
    if case["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = turned.chunk(2, dim=-1)
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, rest], dim=-1)


def plain_attention(s, accumulate):
    """softmax(q K^T / sqrt(D)) V over the rows up to a token's own; requests padded to the longest."""
    case, (r, t) = s["case"], s["new_at"]
    n, hq, hkv, page, most = case["n"], case["hq"], case["hkv"], case["page"], max(s["new"])
    lens, first = torch.tensor(s["lens"], device="cuda"), torch.tensor([a - b for a, b in zip(s["lens"], s["new"])], device="cuda")
    q = torch.zeros(n, most, hq, D, device="cuda")
    q[r, t - first[r]] = s["q"].float()
    q = q.view(n, most, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1, D)           # [n, hkv, group * new, D]
    k, v = (s[x][s["table"].long()].permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, D).float() for x in ("cache_k", "cache_v"))
    j = torch.arange(k.shape[2], device="cuda")
    seen = j <= (first[:, None] + torch.arange(most, device="cuda"))[..., None]                     # [n, new, rows]
    v = v.masked_fill((j >= lens[:, None])[:, None, :, None], 0.0)
    logits = (torch.matmul(q, k.transpose(2, 3)) / math.sqrt(D)).view(n, hkv, hq // hkv, most, -1)
    logits.masked_fill_(~seen[:, None, None], -math.inf)
    top = logits.amax(-1, keepdim=True)
    weight = logits.sub_(top).exp_()
    total = weight.sum(-1, keepdim=True)
    out = torch.matmul(weight.view(n, hkv, -1, k.shape[2]), v).view(n, hkv, -1, most, D) / total
    s["out"].copy_(out.permute(0, 3, 1, 2, 4).reshape(n, most, hq, D)[r, t - first[r]])
    lse = (top + total.log())[..., 0].permute(1, 2, 0, 3).reshape(hq, n, most)
    s["lse"].copy_(lse[:, r, t - first[r]])
    if accumulate:
        r, t = s["row_at"]
        share = (weight / total).sum((2, 3)).permute(0, 2, 1)                                       # [n, rows, hkv]
        s["mass"][s["table"][r, t // page].long(), :, t % page] += share[r, t]


def plain_evict(s):
    """The last `window` rows and the heaviest others, lowest index first among equals, moved to the front."""
    page, hkv = s["case"]["page"], s["case"]["hkv"]
    mass = s["mass"][s["table"].long()].permute(0, 2, 1, 3).flatten(2)                              # [n, hkv, rows]
    budget, window, length = (x[:, None, None] for x in (s["budget"], s["window"], s["len"]))
    window = torch.minimum(window, budget)
    j = torch.arange(mass.shape[2], device="cuda")
    value = mass.masked_fill(j >= length, -math.inf).masked_fill((j >= length - window) & (j < length), math.inf)
    order = torch.sort(value, dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, j.expand_as(order))
    kept = torch.sort((rank >= budget).int(), dim=-1, stable=True).indices                          # kept ones first, ascending
    r, t = index_within(budget.flatten())
    source, heads = kept[r, :, t], torch.arange(hkv, device="cuda")                                 # [sum of budgets, hkv]
    at = s["table"][r[:, None], source // page].long(), heads, source % page
    to = s["out_table"][r, t // page].long()[:, None], heads, (t % page)[:, None]
    rows = s["cache_k"][at], s["cache_v"][at], s["mass"][at]
    s["out_k"][to], s["out_v"][to], s["out_mass"][to] = rows
    # the lists of a request's heads one after another
    first = torch.cumsum(s["budget"], 0) - s["budget"]
    s["kept"][(hkv * first[r] + t)[:, None] + heads * s["budget"][r][:, None]] = source.int()


def index_within(counts):
    """Owner and number within it of `counts` things."""
    r = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), counts)
    return r, torch.arange(len(r), device="cuda") - (torch.cumsum(counts, 0) - counts)[r]


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    """Bytes: every input read once, every output written once.  Operations: Q K^T and P V of the pairs of query and
    row that attend."""
    hq, hkv, (new, lens) = case["hq"], case["hkv"], sizes_of(case)
    row, total, rows = 2 * D, sum(new), sum(lens)          # bytes of one bf16 row
    if case["kind"] == "append":
        moved = 2 * total * (hq + 2 * hkv) * row + total * (4 + 4 * hkv)
        return {"bytes": moved, "flops": total * (hq + hkv) * ((4 * D if case["norm"] else 0) + 3 * case["rotary"])}
    if case["kind"] == "evict":
        kept = sum(budgets_of(case, lens))
        return {"bytes": hkv * (4 * rows + kept * (4 * row + 4 + 4)), "flops": 0}
    pairs = sum(a * (b - a) + a * (a + 1) // 2 for a, b in zip(new, lens))
    moved = 2 * rows * hkv * row + total * hq * (2 * row + 4) + (8 * rows * hkv if case["kind"] == "step" else 0)
    return {"bytes": moved, "flops": 4 * D * hq * pairs}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    page, (new, lens), hq, hkv = case["page"], sizes_of(case), case["hq"], case["hkv"]
    table = s["table"].cpu().tolist()

    def place(tab, r, t):
        return tab[r][t // page], t % page

    def rows(x, r, h, k):
        """Rows 0 .. k - 1 of head h of request r."""
        return torch.cat([x[p, h] for p in table[r][:-(-k // page)]])[:k].double()

    if case["kind"] == "append":
        q, ck, cv, m = s["q"].double(), s["cache_k"].double(), s["cache_v"].double(), s["mass"].double()
        k, half = s["k"].double(), case["rotary"] // 2
        for x, w in ((q, s["q_weight"]), (k, s["k_weight"])):
            if w is not None:
                x /= (torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / D + EPS) ** 0.5
                x *= w.double()
            z = x[..., :2 * half].reshape(*x.shape[:2], half, 2) if case["interleaved"] else \
                torch.stack([x[..., :half], x[..., half:2 * half]], dim=-1)
            turn = torch.polar(torch.ones(half, dtype=torch.float64, device="cuda"),
                               s["positions"].double()[:, None] * torch.tensor(s["inv_freq"], dtype=torch.float64, device="cuda"))
            z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn[:, None])
            x[..., :2 * half] = z.reshape(*x.shape[:2], 2 * half) if case["interleaved"] else torch.cat([z[..., 0], z[..., 1]], -1)
        for r in range(case["n"]):
            t = torch.arange(lens[r] - new[r], lens[r], device="cuda")
            p, o, mine = s["table"][r].long()[t // page], t % page, slice(s["cu"][r], s["cu"][r + 1])
            ck[p, :, o], cv[p, :, o], m[p, :, o] = k[mine], s["v"][mine].double(), 0.0
        return {"q": q, "cache_k": ck, "cache_v": cv, "mass": m}
    if case["kind"] == "evict":
        out_k, out_v, out_m = s["out_k"].double(), s["out_v"].double(), s["out_mass"].double()
        old_k, old_v, kept = s["cache_k"].double(), s["cache_v"].double(), []
        out_table = s["out_table"].cpu().tolist()
        for r in range(case["n"]):
            b, w = s["budgets"][r], min(s["windows"][r], s["budgets"][r])
            pages, to = (torch.tensor([x[r][i // page] for i in range(m)], device="cuda") for x, m in ((table, lens[r]), (out_table, b)))
            for h in range(hkv):
                m = rows(s["mass"], r, h, lens[r]).cpu().tolist()
                best = sorted(range(lens[r] - w), key=lambda i: (-m[i], i))[:b - w]
                mine = torch.tensor(sorted(best) + list(range(lens[r] - w, lens[r])), device="cuda")
                o = torch.arange(b, device="cuda") % page
                out_k[to, h, o], out_v[to, h, o] = old_k[pages[mine], h, mine % page], old_v[pages[mine], h, mine % page]
                out_m[to, h, o] = s["mass"][pages[mine], h, mine % page].double()
                kept.append(mine.int())
        return {"out_k": out_k, "out_v": out_v, "out_mass": out_m, "kept": torch.cat(kept)}
    out = torch.zeros(sum(new), hq, D, dtype=torch.float64, device="cuda")
    lse, m, g = torch.zeros(hq, sum(new), dtype=torch.float64, device="cuda"), s["mass"].double(), hq // hkv
    for r in range(case["n"]):
        mine = slice(s["cu"][r], s["cu"][r + 1])
        at = torch.arange(lens[r], device="cuda")
        p, o = s["table"][r].long()[at // page], at % page
        for h in range(hq):
            logits = s["q"][mine, h].double() @ rows(s["cache_k"], r, h // g, lens[r]).T * D ** -0.5
            logits += torch.full_like(logits, -math.inf).triu(lens[r] - new[r] + 1)
            lse[h, mine] = torch.logsumexp(logits, -1)
            weight = torch.exp(logits - lse[h, mine][:, None])
            out[mine, h] = weight @ rows(s["cache_v"], r, h // g, lens[r])
            if case["kind"] == "step":
                m[p, h // g, o] += weight[0]
    return {"out": out, "lse": lse, **({"mass": m} if case["kind"] == "step" else {})}
