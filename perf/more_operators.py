"""Decoding with beams beside an encoder, as a loop over the paged cache does it: the best continuations of every request's hypotheses out of their
logits, the hypotheses' cached states put in the order of the chosen ones, and attention of decoder tokens to an encoder's states of another
length, which the hypotheses of a request share.

A case is a dict of plain values:

  call            "select" | "reorder" | "cross"
  batch, beams    requests; hypotheses of each
select
  vocab, out      tokens; candidates of each request that are wanted
  dtype           "bf16" | "f32" of the logits
  pad             elements between the end of a row of logits and the next row
  finished        whether some hypotheses have ended: their one continuation is a token that changes nothing
  first           whether this is the first step: the hypotheses but one of each request are not there yet (score -inf)
reorder
  kv_heads, dim, pages ("bf16" | "f32" | "int4"), group, page_rows    the pages' format, as in operators.py
  rows            rows of the longest sequence
  ragged          whether the requests differ in rows
  survivors       hypotheses of each request that have successors
  layers          layers whose pages are brought in order
cross
  heads, kv_heads, dim, dtype     of queries, states and results
  tokens          query tokens of each hypothesis
  rows            rows of the longest source
  ragged          whether the sources differ in rows and, with several tokens, the hypotheses in tokens
  empty           whether a source has no rows at all
  per_head        whether the KV heads of a source differ in rows, as an eviction with budgets leaves them
"""
import functools
import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
PAD_TOKEN = 1


def _select(batch, beams, vocab, out, dtype="bf16", pad=0, finished=False, first=False, name=None):
    c = {"call": "select", "batch": batch, "beams": beams, "vocab": vocab, "out": out, "dtype": dtype, "pad": pad, "finished": finished, "first": first}
    return dict(c, name=name) if name else c


def _reorder(batch, beams, rows, survivors, layers=1, pages="bf16", group=0, page_rows=64, kv_heads=8, dim=128, ragged=False, name=None):
    c = {"call": "reorder", "batch": batch, "beams": beams, "rows": rows, "survivors": survivors, "layers": layers, "pages": pages, "group": group,
         "page_rows": page_rows, "kv_heads": kv_heads, "dim": dim, "ragged": ragged}
    return dict(c, name=name) if name else c


def _cross(batch, beams, tokens, rows, heads=32, kv_heads=8, dim=128, dtype="bf16", ragged=False, empty=False, per_head=False, name=None):
    c = {"call": "cross", "batch": batch, "beams": beams, "tokens": tokens, "rows": rows, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
         "ragged": ragged, "empty": empty, "per_head": per_head}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one step of one request with four hypotheses, twice as many candidates as hypotheses since some may end: the smallest call
        _select(1, 4, 32000, 8, name="select_token"),
        # requests in the middle of their search, some hypotheses ended, logits in fp32, a vocabulary of odd size in rows without padding
        _select(16, 5, 50257, 10, dtype="f32", finished=True, name="select_batch"),
        # a full server: 512 rows of a large vocabulary
        _select(64, 8, 131072, 16, name="select_large"),
        # the cache of one request after such a step, one layer
        _reorder(1, 4, 2085, 2, name="reorder_token"),
        # the caches of a batch, all layers of a small model in one call
        _reorder(8, 8, 2040, 3, layers=8, ragged=True, name="reorder_layers"),
        # one decoder token of four hypotheses over an encoder's 1500 rows
        _cross(1, 4, 1, 1500, name="cross_token"),
        # the same for a batch of sources of different lengths, heads of 64 that share nothing
        _cross(16, 5, 1, 4093, heads=16, kv_heads=16, dim=64, ragged=True, name="cross_batch"),
        # one token of four hypotheses over a long source
        _cross(1, 4, 1, 131072, name="cross_long"),
        # a long decoder prompt over a long source
        _cross(1, 1, 2048, 8192, name="cross_prompt"),
        # decoder prompts of a batch, lengths differ on both sides
        _cross(8, 1, 509, 6001, heads=12, kv_heads=4, ragged=True, name="cross_prompts"),
        # single precision, a few tokens at a time
        _cross(2, 3, 4, 1024, heads=8, kv_heads=2, dim=64, dtype="f32", name="cross_f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["select", "select", "reorder", "token", "token", "token", "prompt", "f32"])
    if kind == "select":
        beams, dtype = rng.randint(1, 16), rng.choice(["bf16", "bf16", "f32"])
        vocab = _log(rng, 1000, 131072)
        batch = _log(rng, 1, max(1, min(64, (1 << 26) // (beams * vocab) // (2 if dtype == "f32" else 1))))
        return _select(batch, beams, vocab, min(32, beams * rng.choice([1, 2, 2])), dtype, pad=rng.choice([0, 0, -vocab % 8, 5]), finished=rng.random() < 0.5,
                       first=rng.random() < 0.15)
    if kind == "reorder":
        pages = rng.choice(["bf16", "bf16", "f32", "int4"])
        kv_heads, dim = rng.choice([(8, 128), (8, 128), (4, 128), (2, 64)])
        beams = rng.randint(2, 8)
        return _reorder(rng.choice([1, 2, 4, 8]), beams, _log(rng, 16, 2048), rng.randint(1, beams), rng.randint(1, 4 if pages == "f32" else 8), pages,
                        rng.choice([32, 64]) if pages == "int4" else 0, rng.choice([16, 32, 64]), kv_heads, dim, rng.random() < 0.6)
    beams = rng.choice([1, 1, 2, 3, 4, 5, 8])
    ragged, none, per_head = rng.random() < 0.6, rng.random() < 0.25, rng.random() < 0.2
    heads, kv_heads, dim = rng.choice([(32, 8, 128), (32, 8, 128), (12, 4, 128), (16, 16, 64), (8, 2, 64)])
    if kind == "f32":
        batch = rng.choice([1, 2, 4])
        return _cross(batch, beams, _log(rng, 1, 16), _log(rng, 50, 2048), 8, 2, 64, "f32", ragged, none and batch > 1, per_head)
    if kind == "token":
        batch = rng.choice([1, 1, 2, 4, 8, 16])
        return _cross(batch, beams, rng.choice([1, 1, 1, 2, 5]), _log(rng, 100, 131072 * 8 // (batch * kv_heads)), heads, kv_heads, dim, "bf16", ragged, none and batch > 1, per_head)
    batch = rng.choice([1, 2, 4, 8])
    tokens = _log(rng, 33, 2048 // batch)
    return _cross(batch, 1, tokens, _log(rng, 100, 8192), heads, kv_heads, dim, "bf16", ragged, none and batch > 1, per_head)


# ---- sizes that follow from a case -----------------------------------------------------------------------------------------------

def _down(most, count, i, ragged):
    return most - (3 * most * i // (4 * max(1, count - 1)) if ragged else 0)


def _source_rows(case):
    """Rows of each source, or of each of its KV heads."""
    S, H = case["batch"], case["kv_heads"]
    rows = [_down(case["rows"], S, i, case["ragged"]) for i in range(S)]
    if case["empty"]:
        rows[-1] = 0
    return [[n * (2 * H - h) // (2 * H) for h in range(H)] for n in rows] if case["per_head"] else rows


def _counts(case):
    """Query tokens of each hypothesis."""
    b = case["batch"] * case["beams"]
    return [_down(case["tokens"], b, i, case["ragged"]) for i in range(b)]


def _lengths(case):
    """Rows of each request's sequences."""
    return [_down(case["rows"], case["batch"], i, case["ragged"]) for i in range(case["batch"])]


def _page_shape(case):
    """Of one head's rows of a page, in elements."""
    if case["pages"] == "int4":
        return (case["page_rows"] // 16, 8 * case["dim"] + 64 * (case["dim"] // case["group"]))
    return (case["page_rows"], case["dim"])


# ---- inputs ------------------------------------------------------------------------------------------------------------------------

def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def prepare(case, seed):
    g = torch.Generator(DEVICE).manual_seed(seed)
    return {"select": _prepare_select, "reorder": _prepare_reorder, "cross": _prepare_cross}[case["call"]](case, g)


def _prepare_select(case, g):
    b, k, v = case["batch"], case["beams"], case["vocab"]
    logits = torch.empty(b * k, v + case["pad"], dtype=TYPES[case["dtype"]], device=DEVICE).normal_(generator=g)
    logits *= 2.5                                    # a few tokens stand out, as in a model's logits
    logits[:, 0] = -math.inf                         # a token that may not be generated
    scores = -20.0 * torch.rand(b, k, generator=g, device=DEVICE)
    if case["first"]:
        scores[:, 1:] = -math.inf
    finished = (torch.rand(b, k, generator=g, device=DEVICE) < 0.25) & (torch.arange(k, device=DEVICE) > 0) if case["finished"] else None
    return {"case": case, "logits": logits[:, :v], "scores": scores, "finished": finished.to(torch.uint8) if case["finished"] else None,
            "parents": torch.zeros(b, case["out"], dtype=torch.int32, device=DEVICE), "tokens": torch.zeros(b, case["out"], dtype=torch.int32, device=DEVICE),
            "best": torch.zeros(b, case["out"], device=DEVICE)}


def _prepare_reorder(case, g):
    b, k, R = case["batch"], case["beams"], case["page_rows"]
    lengths = _lengths(case)
    width = case["rows"] // R + 2
    full = torch.tensor([n // R for n in lengths], device=DEVICE)
    # a request's hypotheses share their first pages and have some of their own at the end
    shared = (full * 3 // 4)[:, None, None]
    ids = torch.randperm(b * (k + 1) * width + 3, generator=g, device=DEVICE)
    private = ids[: b * k * width].view(b, k, width)
    common = ids[b * k * width: b * (k + 1) * width].view(b, 1, width)
    table = torch.where(torch.arange(width, device=DEVICE) < shared, common, private)
    # pages that some table names, closely numbered
    used, table = torch.unique(table, return_inverse=True)
    count = b * k * (width - int(shared.min())) + b * int(shared.max()) + 3
    table = table.view(b * k, width).to(torch.int32)
    order = torch.rand(b, k, generator=g, device=DEVICE).argsort(1)[:, : case["survivors"]]
    pick = torch.randint(0, case["survivors"], (b, k), generator=g, device=DEVICE)
    pick[:, : case["survivors"]] = torch.arange(case["survivors"], device=DEVICE)
    pick = pick.gather(1, torch.rand(b, k, generator=g, device=DEVICE).argsort(1))
    shape = (case["layers"], count, case["kv_heads"], *_page_shape(case))
    if case["pages"] == "int4":
        pools = [torch.empty(shape, dtype=torch.uint8, device=DEVICE).random_(0, 256, generator=g) for _ in range(2)]
    else:
        pools = [torch.empty(shape, dtype=TYPES[case["pages"]], device=DEVICE).normal_(generator=g) for _ in range(2)]
    return {"case": case, "lengths": _int32([n for n in lengths for _ in range(k)]), "table": table, "parents": order.gather(1, pick).to(torch.int32).contiguous(),
            "K": pools[0], "V": pools[1], "table_out": torch.zeros_like(table), "copies": torch.zeros(b * k, 3, dtype=torch.int32, device=DEVICE),
            "dropped": torch.zeros_like(table)}


def _prepare_cross(case, g):
    S, t, Hq, Hkv, d, dtype = case["batch"], case["tokens"], case["heads"], case["kv_heads"], case["dim"], TYPES[case["dtype"]]
    b = S * case["beams"]
    spread = torch.ones(d, device=DEVICE)
    spread[5::32] = 3.0                              # some channels of keys are larger, as a model's are
    # keys and values as one projection of the encoder's states leaves them
    kv = torch.empty(S, case["rows"], 2 * Hkv, d, dtype=dtype, device=DEVICE).normal_(generator=g).transpose(1, 2)
    kv[:, :Hkv] *= spread.to(dtype)
    Q = torch.randn(b, t, Hq, d, generator=g, device=DEVICE).to(dtype).transpose(1, 2)
    counts = _counts(case)
    return {"case": case, "Q": Q, "K": kv[:, :Hkv], "V": kv[:, Hkv:], "lengths": _int32(_source_rows(case)), "counts": _int32(counts) if min(counts) < t else None,
            "out": torch.zeros(b, Hq, t, d, dtype=dtype, device=DEVICE), "lse": torch.zeros(b, Hq, t, device=DEVICE)}


# ---- the framework's calls -----------------------------------------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _handle():
    from paper_2605_08840_b200 import binding as rk
    return rk, rk.Handle()


def _plan(st):
    """The description of the call's sizes and a workspace, which a program keeps from call to call."""
    if "plan" not in st:
        rk, h = _handle()
        case = st["case"]
        dtype = rk.F32 if case.get("dtype") == "f32" else rk.BF16
        if case["call"] == "select":
            desc = rk.make_beams(case["batch"], case["beams"], case["vocab"], case["out"], dtype=dtype, stride=case["vocab"] + case["pad"], pad_token=PAD_TOKEN)
            size = h.beam_workspace_bytes(desc)
        elif case["call"] == "reorder":
            fmt = {"bf16": rk.PAGES_BF16, "f32": rk.PAGES_F32, "int4": rk.PAGES_INT4}[case["pages"]]
            desc = rk.make_paged(case["batch"] * case["beams"], case["kv_heads"], case["kv_heads"], case["dim"], page_format=fmt, page_rows=case["page_rows"],
                                 n_pages=st["K"].shape[1], table_width=st["table"].shape[1], group=case["group"],
                                 dtype=rk.F32 if case["pages"] == "f32" else rk.BF16)
            size = 0
        else:
            desc = rk.make_cross(case["batch"], case["beams"], case["heads"], case["kv_heads"], case["dim"], case["rows"], dtype=dtype, lengths_per_head=case["per_head"])
            size = h.cross_workspace_bytes(desc, case["tokens"])
        st["plan"] = h, desc, torch.empty(size, dtype=torch.uint8, device=DEVICE)
    return st["plan"]


def _run_own(st):
    h, desc, workspace = _plan(st)
    case = st["case"]
    if case["call"] == "select":
        h.beam_select(desc, st["logits"], st["scores"], st["parents"], st["tokens"], st["best"], workspace, finished=st["finished"])
        return {"parents": st["parents"], "tokens": st["tokens"], "scores": st["best"]}
    if case["call"] == "reorder":
        h.paged_reorder(desc, case["beams"], st["parents"], st["lengths"], st["table"], st["table_out"], st["copies"], dropped=st["dropped"])
        h.paged_copy(desc, st["copies"], st["K"], st["V"], n_layers=case["layers"])
        return {"table": st["table_out"], "copies": st["copies"], "dropped": st["dropped"], "K": st["K"], "V": st["V"]}
    h.cross_attend(desc, case["tokens"], st["Q"], st["K"], st["V"], st["out"], workspace, lengths=st["lengths"], lse=st["lse"], counts=st["counts"])
    return {"out": st["out"], "lse": st["lse"]}


# ---- the plain forms -------------------------------------------------------------------------------------------------------------------

def _plain_select(st):
    case = st["case"]
    b, k, n = case["batch"], case["beams"], case["out"]
    x = st["logits"].float()
    x = torch.where(x.isnan(), -math.inf, x).clamp(max=torch.finfo(torch.float32).max) + 0.0
    # the best tokens of every row, ties to the lower one: the bits of a float in an order of integers, the token below them
    bits = x.view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() << 32 | (0x7FFFFFFF - torch.arange(case["vocab"], device=x.device))
    most = min(n, case["vocab"])
    tokens = 0x7FFFFFFF - (key.topk(most, dim=1).values & 0x7FFFFFFF)
    # candidates of different rows lie close together: their scores in 64 bits
    x = x.double()
    top = x.amax(1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    total = top + torch.log(torch.exp(x - top).sum(1, keepdim=True))
    logp = x.gather(1, tokens) - total
    before = st["scores"].double().view(b * k, 1)
    scores = before + logp
    # a hypothesis that is not there has continuations of score -inf, the lower token first as in every tie
    tokens = torch.where(before == -math.inf, torch.arange(most, device=x.device), tokens)
    there = torch.ones_like(tokens, dtype=torch.bool)
    if st["finished"] is not None:
        ended = st["finished"].view(b * k, 1) != 0
        only = torch.arange(most, device=x.device) == 0
        scores = torch.where(ended, before, scores)
        tokens = torch.where(ended, PAD_TOKEN, tokens)
        there = ~ended | only
    scores = torch.where(scores.isnan(), -math.inf, scores)
    # of all rows of a request: the higher score, then the lower row; what is not there comes last
    scores, there, tokens = (z.expand(b * k, most).reshape(b, k * most) for z in (scores, there, tokens))
    best, at = torch.where(there, scores, -math.inf).sort(dim=1, descending=True, stable=True)
    late = (~there.gather(1, at)).int().argsort(dim=1, stable=True)
    at, best = at.gather(1, late)[:, :n], best.gather(1, late)[:, :n]
    return {"parents": (at // most).to(torch.int32), "tokens": tokens.gather(1, at).to(torch.int32), "scores": best.float()}


def _plain_reorder(st):
    case = st["case"]
    b, k, R, W = case["batch"], case["beams"], case["page_rows"], st["table"].shape[1]
    parents, table, n = st["parents"].long(), st["table"].view(b, k, W), st["lengths"].view(b, k)[:, :1].long()
    i = torch.arange(k, device=n.device)
    same = parents[:, :, None] == parents[:, None, :]
    heir = ~(same & (i[None, :] < i[:, None])).any(2)                 # the first successor of its parent
    alive = (parents[:, :, None] == i).any(1)
    dead = alive.int().argsort(dim=1, stable=True)                        # those without successors first
    donor = torch.where(heir, parents, dead.gather(1, ((~heir).cumsum(1) - 1).clamp(min=0)))
    rows_of = lambda who: table.gather(1, who[:, :, None].expand(b, k, W))  # noqa: E731
    full, rest = n // R, (n % R).expand(b, k)
    shared = torch.arange(W, device=n.device) < full[:, :, None]
    from_parent, from_donor = rows_of(parents), rows_of(donor)
    at = full[:, :, None].expand(b, k, 1)
    copy = (donor != parents) & (rest > 0)
    copies = torch.stack([from_parent.gather(2, at)[..., 0], from_donor.gather(2, at)[..., 0], rest.to(torch.int32)], -1)
    copies = torch.where(copy[..., None], copies, _int32([-1, -1, 0]))
    # full pages that no hypothesis names any more, each once
    still = (table[:, :, None, :] == from_parent[:, None, :, :]).any(2)
    again = ((table[:, :, None, :] == table[:, None, :, :]) & (i[None, :] < i[:, None])[:, :, None]).any(2)
    dropped = torch.where(shared & ~still & ~again, table, -1)
    src, dst, rest = copies[copy].long().unbind(-1)
    blocks = (rest + 15) // 16 if case["pages"] == "int4" else rest
    there = (torch.arange(_page_shape(case)[0], device=n.device) < blocks[:, None])[None, :, None, :, None]
    for pool in (st["K"], st["V"]):
        pool[:, dst] = torch.where(there, pool[:, src], pool[:, dst])
    return {"table": torch.where(shared, from_parent, from_donor).view(b * k, W), "copies": copies.view(b * k, 3), "dropped": dropped.view(b * k, W), "K": st["K"], "V": st["V"]}


def _plain_cross(st):
    case = st["case"]
    S, k, Hkv, t, d = case["batch"], case["beams"], case["kv_heads"], case["tokens"], case["dim"]
    G = case["heads"] // Hkv
    q = st["Q"].float().reshape(S, k, Hkv, G, t, d).transpose(1, 2).reshape(S, Hkv, k * G * t, d)
    s = q @ st["K"].float().transpose(2, 3) / math.sqrt(d)
    lengths = st["lengths"].view(S, -1, 1, 1)
    s = torch.where(torch.arange(case["rows"], device=s.device) < lengths, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    out = p @ st["V"].float() / torch.where(total > 0, total, 1.0)
    out, lse = (z.view(S, Hkv, k, G, t, -1).transpose(1, 2).reshape(S * k, Hkv * G, t, -1) for z in (out, top + torch.log(total)))
    if st["counts"] is not None:
        there = (torch.arange(t, device=s.device) < st["counts"][:, None])[:, None, :, None]
        out, lse = torch.where(there, out, 0.0), torch.where(there, lse, -math.inf)
    return {"out": out.to(TYPES[case["dtype"]]), "lse": lse[..., 0]}


def run(st):
    if own:
        return _run_own(st)
    return {"select": _plain_select, "reorder": _plain_reorder, "cross": _plain_cross}[st["case"]["call"]](st)


def work(case):
    """Every input read once, every output written once."""
    b, k = case["batch"], case["beams"]
    if case["call"] == "select":
        es = 4 if case["dtype"] == "f32" else 2
        live = b * (1 if case["first"] else k)
        return {"bytes": live * case["vocab"] * es + b * k * 4 + b * case["out"] * 12, "flops": 4 * live * case["vocab"]}
    if case["call"] == "reorder":
        R, W = case["page_rows"], case["rows"] // case["page_rows"] + 2
        size = 2 if case["pages"] == "bf16" else 4 if case["pages"] == "f32" else 1
        rows = sum((n % R + 15) // 16 if case["pages"] == "int4" else n % R for n in _lengths(case))
        moved = (k - case["survivors"]) * rows * case["kv_heads"] * _page_shape(case)[1] * size
        return {"bytes": 2 * 2 * case["layers"] * moved + 3 * 4 * b * k * W + b * k * 20, "flops": 0}
    es = 4 if case["dtype"] == "f32" else 2
    rows, counts = _source_rows(case), _counts(case)
    each = [sum(n) if case["per_head"] else n * case["kv_heads"] for n in rows]
    tokens = [sum(counts[i * k:(i + 1) * k]) for i in range(b)]
    G, d = case["heads"] // case["kv_heads"], case["dim"]
    return {"bytes": 2 * sum(each) * d * es + b * k * case["heads"] * case["tokens"] * (d * es + 4) + sum(counts) * case["heads"] * d * es,
            "flops": 4 * G * d * sum(n * t for n, t in zip(each, tokens))}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return {"select": _exact_select, "reorder": _exact_reorder, "cross": _exact_cross}[case["call"]](case, st)


def _exact_select(case, st):
    b, k, v, n = case["batch"], case["beams"], case["vocab"], case["out"]
    got = {"parents": [], "tokens": [], "scores": []}
    for i in range(b):
        x = st["logits"][i * k:(i + 1) * k].double()
        scores = st["scores"][i].double()[:, None] + torch.log_softmax(x, 1)
        if st["finished"] is not None:
            ended = st["finished"][i] != 0
            scores[ended] = -math.inf
            scores[ended, PAD_TOKEN] = st["scores"][i][ended].double()
        order = scores.flatten().argsort(descending=True, stable=True)[:n]
        got["parents"].append(order // v)
        got["tokens"].append(order % v)
        got["scores"].append(scores.flatten()[order])
    return {"parents": torch.stack(got["parents"]).to(torch.int32), "tokens": torch.stack(got["tokens"]).to(torch.int32), "scores": torch.stack(got["scores"])}


def _exact_reorder(case, st):
    b, k, R = case["batch"], case["beams"], case["page_rows"]
    old, parents = st["table"].view(b, k, -1).tolist(), st["parents"].tolist()
    table, copies, dropped = [], [], []
    K, V = (p if case["pages"] == "int4" else p.double() for p in (st["K"], st["V"]))
    for i, n in enumerate(_lengths(case)):
        full, rest = divmod(n, R)
        free = [j for j in range(k) if j not in parents[i]]
        taken = set()
        for j in range(k):
            p = parents[i][j]
            donor = free.pop(0) if p in taken else p
            taken.add(p)
            table.append(old[i][p][:full] + old[i][donor][full:])
            if donor != p and rest:
                copies.append([old[i][p][full], old[i][donor][full], rest])
                many = -(-rest // 16) if case["pages"] == "int4" else rest
                for pool in (K, V):
                    pool[:, copies[-1][1], :, :many] = pool[:, copies[-1][0], :, :many]
            else:
                copies.append([-1, -1, 0])
        named = [set(old[i][p][c] for p in parents[i]) for c in range(full)]
        for j in range(k):
            row = [-1] * len(old[i][j])
            for c in range(full):
                if old[i][j][c] not in named[c]:
                    row[c] = old[i][j][c]
                    named[c].add(row[c])
            dropped.append(row)
    return {"table": _int32(table), "copies": _int32(copies), "dropped": _int32(dropped), "K": K, "V": V}


def _exact_cross(case, st):
    S, k, G = case["batch"], case["beams"], case["heads"] // case["kv_heads"]
    rows, counts = _source_rows(case), _counts(case)
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full(st["lse"].shape, -math.inf, dtype=torch.float64, device=DEVICE)
    for i in range(S * k):
        for h in range(case["heads"]):
            n = rows[i // k][h // G] if case["per_head"] else rows[i // k]
            c = counts[i]
            if n == 0 or c == 0:
                continue
            K, V = (st[x][i // k, h // G, :n].double() for x in ("K", "V"))
            s = st["Q"][i, h, :c].double() @ K.T / math.sqrt(case["dim"])
            lse[i, h, :c] = torch.logsumexp(s, -1)
            out[i, h, :c] = torch.softmax(s, -1) @ V
    return {"out": out, "lse": lse}
