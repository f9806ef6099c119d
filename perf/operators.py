"""The paged cache behind an eviction, as a decoding loop uses it: keys and values appended to pages with the position
rotation applied on the way, attention over the pages (16 or 32 bits, or 4 bits with group scales; scores optionally capped by
a tanh), and rows read back out of the pages for the next eviction.

A case is a dict of plain values:

  call            "append" | "attend" | "read"
  heads, kv_heads, dim, dtype     query heads, KV heads, head_dim; "bf16" | "f32" for what goes in and comes out
  pages           "bf16" | "f32" | "int4"
  group           dims that share a step and an offset ("int4"; else 0)
  page_rows       rows of a page
  batch, tokens   sequences; new tokens of each (append), query tokens of each (attend)
  rows            rows of the longest sequence, the new ones included
  ragged          whether the sequences differ in rows and, with several tokens, in tokens
  rotary          dims that are rotated (0: none, keys of an evicted cache carry their rotation)
  interleaved     pairs (2i, 2i + 1) instead of (i, i + rotary / 2)
  softcap         0, or the cap of the scores

Page layout.  "bf16", "f32": [pages, kv_heads, page_rows, dim].  "int4": [pages, kv_heads, page_rows / 16, bytes] of uint8; such
a block of 16 rows has their codes, dim / 2 bytes each, and then for every group 64 bytes: for c = 0..3 the steps of the rows c,
c + 4, c + 8, c + 12 and then their offsets, all bf16.  The codes of a row lie in an order of their own: in K, 32-bit word
c * (dim / 32) + g has dims 32 g + 8 c + (0..7) from its lowest 4 bits on; in V, 16-bit unit r * (dim / 32) + g has dims
32 g + 4 r + (0..3).  A value is offset + step * code; offset is the group's minimum rounded down to bf16, step a fifteenth of
the range above it rounded up to bf16, a code the nearest one (ties to even).
"""
import functools
import math

import torch

own = False

DEVICE = "cuda"
POSITIONS = 132096          # of the rotation tables
BASE = 500000.0             # of the rotation's frequencies
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(call, pages, batch, tokens, rows, group=0, ragged=False, rotary=0, interleaved=False, softcap=0.0, page_rows=64, heads=32, kv_heads=8, dim=128,
          dtype="bf16", name=None):
    c = {"call": call, "pages": pages, "batch": batch, "tokens": tokens, "rows": rows, "group": group, "ragged": ragged, "rotary": rotary,
         "interleaved": interleaved, "softcap": softcap, "page_rows": page_rows, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one generated token of one sequence after an eviction: once per layer and token, the smallest call
        _case("append", "bf16", 1, 1, 2085, rotary=128, name="append_token"),
        # the rows that an eviction kept go into 4-bit pages; their keys are rotated already
        _case("append", "int4", 1, 2048, 2048, group=64, name="append_compacted"),
        # a batch of prompts of different lengths, half of the dims rotated, in interleaved pairs
        _case("append", "bf16", 8, 4093, 4093, ragged=True, rotary=64, interleaved=True, page_rows=16, name="append_prompts"),
        # a long prompt into 4-bit pages with fine groups
        _case("append", "int4", 1, 32768, 32768, group=32, rotary=128, name="append_long_prompt"),
        # one decode step over a compacted 4-bit cache that has grown by some tokens
        _case("attend", "int4", 1, 1, 2085, group=64, name="attend_compacted"),
        # the same for a batch of sequences
        _case("attend", "int4", 8, 1, 2176, group=64, name="attend_compacted_batch"),
        # one decode step over a whole long cache in 4 bits
        _case("attend", "int4", 1, 1, 131072, group=64, page_rows=256, name="attend_full"),
        # a decode step of sequences of different lengths over bf16 pages, scores capped
        _case("attend", "bf16", 8, 1, 32768, ragged=True, softcap=50.0, page_rows=16, name="attend_ragged_capped"),
        # the tiny single-precision workload
        _case("attend", "f32", 1, 1, 1024, heads=8, kv_heads=2, dim=64, dtype="f32", page_rows=32, name="attend_f32_tiny"),
        # the next turn of a conversation: a chunk of prompt over a 4-bit cache and itself
        _case("attend", "int4", 1, 2048, 18432, group=128, softcap=30.0, name="attend_chunk"),
        # a compacted cache is read back for the eviction that comes after 128 generated tokens
        _case("read", "int4", 1, 0, 2176, group=64, name="read_compacted"),
        # whole sequences are read back for their first eviction
        _case("read", "int4", 8, 0, 32749, group=32, ragged=True, name="read_batch"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "attend", "attend", "attend", "chunk", "f32", "read"])
    page_rows = rng.choice([16, 32, 64, 128, 256])
    batch = rng.choice([1, 1, 2, 4, 8])
    ragged = batch > 1 and rng.random() < 0.7
    heads, kv_heads, dim = rng.choice([(32, 8, 128), (32, 8, 128), (32, 8, 128), (12, 4, 128), (8, 2, 64)])
    pages = rng.choice(["int4", "int4", "bf16"])
    group = rng.choice([g for g in (32, 64, 128) if g <= dim]) if pages == "int4" else 0
    cap = rng.choice([0.0, 0.0, 30.0, 50.0])
    shape = {"page_rows": page_rows, "ragged": ragged, "heads": heads, "kv_heads": kv_heads, "dim": dim}
    if kind == "f32":
        pages, rows = rng.choice(["f32", "int4"]), _log(rng, 100, 8192)
        shape.update(heads=8, kv_heads=2, dim=64, dtype="f32", group=rng.choice([32, 64]) if pages == "int4" else 0)
        if rng.random() < 0.5:
            tokens = _log(rng, 1, 64)
            return _case("append", pages, batch, tokens, rows + tokens, rotary=rng.choice([0, 32, 64]), **shape)
        return _case("attend", pages, batch, rng.choice([1, 1, 4]), rows, softcap=cap, **shape)
    if kind == "append":
        tokens = rng.choice([1, _log(rng, 2, 32768 // batch), _log(rng, 2, 32768 // batch)])
        before = rng.choice([0, _log(rng, 16, 4096)])
        return _case("append", pages, batch, tokens, before + tokens, group=group, rotary=rng.choice([0, dim // 2, dim, dim]), interleaved=rng.random() < 0.3, **shape)
    if kind == "read":
        return _case("read", pages, batch, 0, _log(rng, 500, 131072 // batch), group=group, **shape)
    if kind == "chunk":
        tokens = _log(rng, 2, 2048 // batch)
        return _case("attend", pages, batch, tokens, tokens + _log(rng, 100, 16384), group=group, softcap=cap, **shape)
    return _case("attend", pages, batch, 1, _log(rng, 500, 131072 // batch), group=group, softcap=cap, **shape)


def _counts(case):
    """New tokens of each sequence."""
    b, t = case["batch"], case["tokens"]
    return [t - (3 * t * i // (4 * (b - 1)) if case["ragged"] else 0) for i in range(b)]


def _lengths(case):
    """Rows of each sequence, the new ones included."""
    b, before = case["batch"], case["rows"] - case["tokens"]
    return [n + before - (3 * before * i // (4 * (b - 1)) if case["ragged"] else 0) for i, n in enumerate(_counts(case))]


# ---- 4-bit rows ------------------------------------------------------------------------------------------------------------

def _round_to_bf16(x, up):
    """x (32 bits) to the nearest bf16 value that is not below (up) or above it."""
    bits = x.contiguous().view(torch.int32)
    toward_zero = bits & -65536
    away = (bits != toward_zero) & ((bits >= 0) == up)
    return torch.where(away, toward_zero + 65536, toward_zero).view(torch.float32)


def _quantise(x, group):
    """(codes, steps, offsets) of rows x [..., dim] in 32 bits; steps and offsets [..., dim / group] are bf16 values in 32 bits."""
    g = x.unflatten(-1, (-1, group))
    lo = _round_to_bf16(g.amin(-1), False)
    span = g.amax(-1) - lo
    step = _round_to_bf16(span / torch.full_like(span, 15.0), True)         # by a tensor: a quotient, not a product with 1 / 15
    scaled = (g - lo[..., None]) / torch.where(step > 0, step, 1.0)[..., None]
    return scaled.round().clamp(0, 15).flatten(-2), step, lo


def _values(codes, step, lo):
    return (codes.unflatten(-1, (step.shape[-1], -1)) * step[..., None] + lo[..., None]).flatten(-2)


def _stored(codes, is_key):
    """Codes [..., dim] in the order in which a row's bytes hold them, two to a byte."""
    dim = codes.shape[-1]
    c = codes.unflatten(-1, (dim // 32, 4, 8) if is_key else (dim // 32, 8, 4)).transpose(-3, -2).reshape(*codes.shape[:-1], dim // 2, 2).to(torch.uint8)
    return c[..., 0] | (c[..., 1] << 4)


def _codes(stored, is_key):
    dim = 2 * stored.shape[-1]
    c = torch.stack([stored & 15, stored >> 4], -1).flatten(-2)
    return c.unflatten(-1, (4, dim // 32, 8) if is_key else (8, dim // 32, 4)).transpose(-3, -2).flatten(-3).to(torch.float32)


def _blocks(rows, group, is_key):
    """The blocks [..., n / 16, bytes] of rows [..., n, dim]."""
    codes, step, lo = _quantise(rows, group)
    n, dim = rows.shape[-2:]
    data = _stored(codes, is_key).unflatten(-2, (n // 16, 16)).flatten(-2)
    both = torch.stack([step, lo], -1).to(torch.bfloat16).unflatten(-3, (n // 16, 4, 4))       # [..., block, row / 4, row % 4, group, 2]
    order = both.movedim(-2, -4).transpose(-3, -2).transpose(-2, -1)                            # [..., block, group, row % 4, 2, row / 4]
    return torch.cat([data, order.contiguous().view(torch.uint8).flatten(-4)], -1)


def _rows_of(blocks, dim, group, is_key):
    """Rows [..., n, dim] in 32 bits of the blocks [..., n / 16, bytes]."""
    codes = _codes(blocks[..., : 8 * dim].unflatten(-1, (16, dim // 2)), is_key)
    both = blocks[..., 8 * dim:].contiguous().view(torch.bfloat16).float().unflatten(-1, (dim // group, 4, 2, 4))
    both = both.transpose(-2, -1).transpose(-3, -2).movedim(-4, -2).flatten(-4, -3)             # [..., block, row, group, 2]
    return _values(codes, both[..., 0], both[..., 1]).flatten(-3, -2)


# ---- inputs ----------------------------------------------------------------------------------------------------------------

def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _new_pages(case, count, g):
    """Pages of K and V that are full of rows.  Keys have some channels of larger spread, as a model's keys do."""
    shape = (count, case["kv_heads"], case["page_rows"], case["dim"])
    spread = torch.ones(case["dim"], device=DEVICE)
    spread[5::32] = 3.0
    K = torch.randn(shape, generator=g, device=DEVICE) * spread
    V = torch.randn(shape, generator=g, device=DEVICE)
    if case["pages"] == "int4":
        return _blocks(K, case["group"], True), _blocks(V, case["group"], False)
    return K.to(TYPES[case["pages"]]), V.to(TYPES[case["pages"]])


def prepare(case, seed):
    g = torch.Generator(DEVICE).manual_seed(seed)
    b, t, Hq, Hkv, d, dtype = case["batch"], case["tokens"], case["heads"], case["kv_heads"], case["dim"], TYPES[case["dtype"]]
    width = -(-case["rows"] // case["page_rows"])
    count = b * width + 3                                          # some pages belong to nobody
    lengths, counts = _lengths(case), _counts(case)
    st = {"case": case, "lengths": _int32(lengths), "counts": _int32(counts) if len(set(counts)) > 1 else None,
          "first": _int32([n - c for n, c in zip(lengths, counts)]),
          "table": torch.randperm(count, generator=g, device=DEVICE)[: b * width].view(b, width).to(torch.int32)}
    st["K_pages"], st["V_pages"] = _new_pages(case, count, g)

    def outputs(*shapes):
        return [torch.zeros(s, dtype=dtype, device=DEVICE) for s in shapes]

    if case["call"] == "read":
        st["K"], st["V"] = outputs(*2 * [(b, Hkv, case["rows"], d)])
        return st
    if case["call"] == "attend":
        st["Q"] = torch.randn(b, t, Hq, d, generator=g, device=DEVICE).to(dtype).transpose(1, 2)
        (st["out"],) = outputs((b, Hq, t, d))
        st["lse"] = torch.zeros(b, Hq, t, device=DEVICE)
        return st
    if case["rotary"]:
        # the queries, keys and values of the new tokens as a projection leaves them
        x = torch.randn(b, t, Hq + 2 * Hkv, d, generator=g, device=DEVICE).to(dtype).transpose(1, 2)
        st["Q"], st["K_new"], st["V_new"] = x.split([Hq, Hkv, Hkv], dim=1)
        (st["Q_out"],) = outputs((b, Hq, t, d))
        angle = torch.arange(POSITIONS, device=DEVICE, dtype=torch.float64)[:, None] * BASE ** (
            -torch.arange(0, case["rotary"], 2, device=DEVICE, dtype=torch.float64) / case["rotary"])
        st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
        start = torch.randint(0, POSITIONS - case["rows"], (b, 1), generator=g, device=DEVICE)     # an evicted cache has fewer rows than positions
        st["positions"] = (start + st["first"][:, None] + torch.arange(t, device=DEVICE)).to(torch.int32)
    else:
        st["K_new"], st["V_new"] = (torch.randn(b, Hkv, t, d, generator=g, device=DEVICE).to(dtype) for _ in range(2))
    if case["pages"] == "int4":
        st["K"], st["V"] = outputs(*2 * [(b, Hkv, t, d)])
    return st


# ---- the framework's calls ---------------------------------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _handle():
    from paper_2605_08840_b200 import binding as rk
    return rk, rk.Handle()


def _plan(st):
    """The cache's description, the rotation tables and a workspace, which a program keeps from call to call."""
    if "plan" not in st:
        rk, h = _handle()
        case = st["case"]
        cache = rk.make_paged(case["batch"], case["heads"], case["kv_heads"], case["dim"], page_format={"bf16": rk.PAGES_BF16, "f32": rk.PAGES_F32, "int4": rk.PAGES_INT4}[case["pages"]],
                              page_rows=case["page_rows"], n_pages=st["K_pages"].shape[0], table_width=st["table"].shape[1], group=case["group"],
                              dtype=rk.F32 if case["dtype"] == "f32" else rk.BF16, softcap=case["softcap"])
        rotation = rk.make_rotation(st["cos"], st["sin"], case["rotary"], interleaved=case["interleaved"]) if "cos" in st else None
        workspace = torch.empty(h.paged_workspace_bytes(cache, max(1, case["tokens"])), dtype=torch.uint8, device=DEVICE)
        st["plan"] = h, cache, rotation, workspace
    return st["plan"]


def _run_own(st):
    h, cache, rotation, workspace = _plan(st)
    case = st["case"]
    pages = st["K_pages"], st["V_pages"], st["lengths"], st["table"]
    if case["call"] == "read":
        h.paged_read(cache, *pages, case["rows"], st["K"], st["V"])
        return {"K": st["K"], "V": st["V"]}
    if case["call"] == "attend":
        h.paged_attend(cache, case["tokens"], st["Q"], *pages, st["out"], workspace, lse=st["lse"], counts=st["counts"])
        return {"out": st["out"], "lse": st["lse"]}
    h.paged_append(cache, case["tokens"], st["K_new"], st["V_new"], *pages, counts=st["counts"], positions=st.get("positions"), rotation=rotation,
                   Q=st.get("Q"), Q_out=st.get("Q_out"))
    got = {"Q": st["Q_out"]} if rotation else {}
    if case["pages"] == "int4":      # what the 4-bit rows stand for
        h.paged_read(cache, *pages, case["tokens"], st["K"], st["V"], first=st["first"])
        return dict(got, K=st["K"], V=st["V"])
    return dict(got, K=st["K_pages"], V=st["V_pages"])


# ---- the plain forms ---------------------------------------------------------------------------------------------------------

def _sequences(pages, table, case, is_key):
    """The rows [b, kv_heads, n, dim] of all sequences in 32 bits, page by page."""
    x = pages[table.long()].transpose(1, 2).flatten(2, 3)
    return _rows_of(x, case["dim"], case["group"], is_key) if case["pages"] == "int4" else x.float()


def _rotate(x, st):
    """x [b, heads, tokens, dim] in 32 bits at the tokens' positions."""
    case = st["case"]
    cos, sin = (st[k][st["positions"].long()][:, None] for k in ("cos", "sin"))
    x, rest = x.split([case["rotary"], case["dim"] - case["rotary"]], dim=-1)
    a, b = x.unflatten(-1, (-1, 2)).unbind(-1) if case["interleaved"] else x.chunk(2, -1)
    turned = [a * cos - b * sin, b * cos + a * sin]
    return torch.cat([torch.stack(turned, -1).flatten(-2) if case["interleaved"] else torch.cat(turned, -1), rest], -1)


def _run_plain(st):
    case, dtype = st["case"], TYPES[st["case"]["dtype"]]
    n = st["lengths"].long()[:, None]
    if case["call"] == "read":
        there = (torch.arange(case["rows"], device=n.device) < n)[:, None, :, None]
        K, V = (_sequences(st[k], st["table"], case, k == "K_pages")[:, :, : case["rows"]] for k in ("K_pages", "V_pages"))
        return {"K": torch.where(there, K, 0.0).to(dtype), "V": torch.where(there, V, 0.0).to(dtype)}
    i = torch.arange(case["tokens"], device=n.device)
    count = st["counts"].long()[:, None] if st["counts"] is not None else torch.full_like(n, case["tokens"])
    if case["call"] == "attend":
        K, V = _sequences(st["K_pages"], st["table"], case, True), _sequences(st["V_pages"], st["table"], case, False)
        G = case["heads"] // case["kv_heads"]
        q = st["Q"].float().unflatten(1, (case["kv_heads"], G)).flatten(2, 3)                      # [b, kv_heads, G * tokens, dim]
        s = (q @ K.transpose(-1, -2)) / math.sqrt(case["dim"])
        if case["softcap"]:
            s = torch.tanh(s / case["softcap"]) * case["softcap"]
        sees = torch.where(i < count, n - (count - 1 - i), 0)                                       # rows that a query token sees
        mask = torch.arange(K.shape[2], device=n.device) < sees[..., None]
        s = s.unflatten(2, (G, -1)).masked_fill(~mask[:, None, None], -math.inf)
        top = s.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, 0.0, top)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        out = (p.flatten(2, 3) @ V).unflatten(2, (G, -1)) / torch.where(total > 0, total, 1.0)
        return {"out": out.flatten(1, 2).to(dtype), "lse": (top + torch.log(total)).squeeze(-1).flatten(1, 2)}
    there = i < count
    K, V, got = st["K_new"].float(), st["V_new"].float(), {}
    if "Q" in st:
        K = _rotate(K, st)
        got["Q"] = torch.where(there[:, None, :, None], _rotate(st["Q"].float(), st), 0.0).to(dtype)
    row = (n - count + i)[there]
    page = st["table"].long()[torch.where(there)[0], row // case["page_rows"]]
    at = row % case["page_rows"]
    new = [x.transpose(1, 2)[there] for x in (K, V)]                                                # [rows, kv_heads, dim]
    if case["pages"] != "int4":
        for pages, x in zip((st["K_pages"], st["V_pages"]), new):
            pages[page, :, at] = x.to(pages.dtype)
        return dict(got, K=st["K_pages"], V=st["V_pages"])
    for name, pages, x in zip(("K", "V"), (st["K_pages"], st["V_pages"]), new):
        codes, step, lo = _quantise(x, case["group"])
        dim, groups = case["dim"], case["dim"] // case["group"]
        block, r = at // 16, at % 16
        byte = torch.arange(dim // 2, device=n.device)
        pages[page[:, None], :, block[:, None], r[:, None] * (dim // 2) + byte] = _stored(codes, name == "K").transpose(1, 2)
        pair = torch.stack([step, lo], -1).to(torch.bfloat16).view(torch.uint8).unflatten(-1, (2, 2))   # [rows, kv_heads, group, step or offset, byte]
        place = (8 * dim + 64 * torch.arange(groups, device=n.device)[:, None, None] + 8 * torch.arange(2, device=n.device)[:, None] + torch.arange(2, device=n.device)).flatten()
        pages[page[:, None], :, block[:, None], (16 * (r % 4) + 2 * (r // 4))[:, None] + place] = pair.flatten(2).transpose(1, 2)
        value = torch.zeros_like(st[name])
        value.transpose(1, 2)[there] = _values(codes, step, lo).to(dtype)
        got[name] = value
    return got


def run(st):
    return _run_own(st) if own else _run_plain(st)


def work(case):
    """Every input read once, every output written once: the rows that are there, as their format holds them."""
    b, Hq, Hkv, d, t = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["tokens"]
    es = 4 if case["dtype"] == "f32" else 2
    row = {"bf16": 2 * d, "f32": 4 * d, "int4": d // 2 + 4 * (d // case["group"] if case["group"] else 0)}[case["pages"]]
    lengths, counts = _lengths(case), _counts(case)
    if case["call"] == "read":
        return {"bytes": 2 * Hkv * (sum(lengths) * row + b * case["rows"] * d * es), "flops": 2 * 2 * Hkv * sum(lengths) * d}
    if case["call"] == "attend":
        pairs = sum(max(0, n - (c - 1 - i)) for n, c in zip(lengths, counts) for i in range(c))
        return {"bytes": 2 * Hkv * sum(lengths) * row + b * Hq * t * (2 * d * es + 4), "flops": 4 * Hq * d * pairs}
    new = sum(counts)
    size = 2 * Hkv * new * (d * es + row)
    if case["rotary"]:
        size += 2 * Hq * new * d * es + new * case["rotary"] * 4
    if case["pages"] == "int4":
        size += 2 * Hkv * new * (row + d * es)
    return {"bytes": size, "flops": new * (3 * (Hq + Hkv) * case["rotary"] + (8 * Hkv * d if case["pages"] == "int4" else 0))}


# ---- the definition in 64 bits -------------------------------------------------------------------------------------------------

def _exact_rows(st, key, b, rows):
    """The first `rows` rows [kv_heads, rows, dim] of sequence b, from the layout as the head of this file states it."""
    case = st["case"]
    R, d = case["page_rows"], case["dim"]
    j = torch.arange(rows, device=DEVICE)
    page, r = st["table"][b].long()[j // R], j % R
    pages = st["K_pages" if key else "V_pages"]
    if case["pages"] != "int4":
        return pages[page, :, r].double().transpose(0, 1)
    block = pages[page, :, r // 16].to(torch.int64).transpose(0, 1)                # [kv_heads, rows, bytes]
    r = r % 16
    dim = torch.arange(d, device=DEVICE)
    if key:
        nibble = 8 * ((dim % 32) // 8 * (d // 32) + dim // 32) + dim % 8
    else:
        nibble = 4 * ((dim % 32) // 4 * (d // 32) + dim // 32) + dim % 4
    at = (r[:, None] * (d // 2) + nibble // 2).expand(block.shape[0], -1, -1)
    code = (block.gather(2, at) >> (4 * (nibble % 2))) & 15

    def bf16(offset):                                                               # two bytes are the upper half of a 32-bit float
        a = (8 * d + 64 * (dim // case["group"]) + offset + (16 * (r % 4) + 2 * (r // 4))[:, None]).expand(block.shape[0], -1, -1)
        return ((block.gather(2, a + 1) << 24) + (block.gather(2, a) << 16)).to(torch.int32).view(torch.float32).double()

    return bf16(8) + bf16(0) * code


def _exact_grid(x, up):
    """x to bf16, down or up, by its exponent."""
    _, e = torch.frexp(x)
    unit = torch.ldexp(torch.ones_like(x), e - 8)
    return (torch.ceil(x / unit) if up else torch.floor(x / unit)) * unit


def _exact_quantised(x, group):
    shape = x.shape
    x = x.reshape(*shape[:-1], shape[-1] // group, group)
    lo = _exact_grid(x.min(-1, keepdim=True).values, False)
    step = _exact_grid((x.max(-1, keepdim=True).values - lo) / 15, True)
    return (lo + step * torch.clamp(torch.round((x - lo) / step), 0, 15)).reshape(shape)


def _exact_rotated(x, st, b):
    case, h = st["case"], st["case"]["rotary"] // 2
    x = x.double().clone()
    i = torch.arange(h, device=DEVICE)
    first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + h)
    z = torch.complex(x[..., first], x[..., second]) * torch.complex(st["cos"].double(), st["sin"].double())[st["positions"][b].long()]
    x[..., first], x[..., second] = z.real, z.imag
    return x


def exact(case, seed):
    st = prepare(case, seed)
    lengths, counts = _lengths(case), _counts(case)
    if case["call"] == "read":
        K, V = (torch.zeros(st["K"].shape, dtype=torch.float64, device=DEVICE) for _ in range(2))
        for b, n in enumerate(lengths):
            K[b, :, :n], V[b, :, :n] = _exact_rows(st, True, b, n), _exact_rows(st, False, b, n)
        return {"K": K, "V": V}
    if case["call"] == "attend":
        out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEVICE)
        lse = torch.full(st["lse"].shape, -math.inf, dtype=torch.float64, device=DEVICE)
        G = case["heads"] // case["kv_heads"]
        for b, (n, c) in enumerate(zip(lengths, counts)):
            K, V = _exact_rows(st, True, b, n), _exact_rows(st, False, b, n)
            for h in range(case["heads"]):
                s = st["Q"][b, h, :c].double() @ K[h // G].T / math.sqrt(case["dim"])
                if case["softcap"]:
                    s = case["softcap"] * torch.tanh(s / case["softcap"])
                hidden = torch.arange(n, device=DEVICE)[None] > (n - c + torch.arange(c, device=DEVICE))[:, None]
                s[hidden] = -math.inf
                lse[b, h, :c] = torch.logsumexp(s, -1)
                out[b, h, :c] = torch.softmax(s, -1) @ V[h // G]
        return {"out": out, "lse": lse}
    got = {}
    if "Q" in st:
        got["Q"] = torch.zeros(st["Q_out"].shape, dtype=torch.float64, device=DEVICE)
    if case["pages"] == "int4":
        got["K"], got["V"] = (torch.zeros(st["K"].shape, dtype=torch.float64, device=DEVICE) for _ in range(2))
    else:
        got["K"], got["V"] = st["K_pages"].double(), st["V_pages"].double()
    for b, (n, c) in enumerate(zip(lengths, counts)):
        K, V = st["K_new"][b].double(), st["V_new"][b].double()
        if "Q" in st:
            got["Q"][b, :, :c] = _exact_rotated(st["Q"][b], st, b)[:, :c]
            K = _exact_rotated(K, st, b)
        if case["pages"] == "int4":
            got["K"][b, :, :c], got["V"][b, :, :c] = _exact_quantised(K, case["group"])[:, :c], _exact_quantised(V, case["group"])[:, :c]
        else:
            j = torch.arange(n - c, n, device=DEVICE)
            page, r = st["table"][b].long()[j // case["page_rows"]], j % case["page_rows"]
            got["K"][page, :, r], got["V"][page, :, r] = K[:, :c].transpose(0, 1), V[:, :c].transpose(0, 1)
    return got
