"""The paged cache: rows appended (with the position rotation), attended over and read back, against plain implementations in
64 bits that are written from the header's formulas and byte layout."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2605_08840_b200 import binding as rk

NEG_INF = float("-inf")


# ---- plain implementations (numpy, 64 bits) -------------------------------------------------------------------------------------

def bf16_round(x):
    """To the nearest bf16 value, ties to even."""
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16).float().numpy()


def bf16_directed(x, up):
    """float32 -> the bf16 value next to it from above or below."""
    r = bf16_round(x)
    wrong = r < x if up else r > x
    bits = r.view(np.int32).astype(np.int64)
    away = bits + 65536                       # one further from zero
    toward = np.where((bits & 0x7FFFFFFF) == 0, np.int64(0x00010000 if up else -0x7FFF0000), bits - 65536)
    nxt = np.where((r > 0) == up, away, toward).astype(np.int64)
    nxt = np.where(r == 0, 0x00010000 if up else 0x80010000 - (1 << 32), nxt)
    return np.where(wrong, nxt.astype(np.int32).view(np.float32), r)


def quantise(x, group):
    """(codes, steps, offsets) of float32 rows [..., d] by the header's rule, in float32 as stated there."""
    x = np.clip(np.nan_to_num(x.astype(np.float32), nan=0.0, posinf=np.float32(2.0 ** 120), neginf=np.float32(-2.0 ** 120)),
                np.float32(-2.0 ** 120), np.float32(2.0 ** 120))
    g = x.reshape(*x.shape[:-1], -1, group)
    lo = bf16_directed(g.min(-1), False)
    step = bf16_directed((g.max(-1) - lo) / np.float32(15), True)
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(step[..., None] > 0, np.rint((g - lo[..., None]) / step[..., None]), 0)
    return np.clip(q, 0, 15).astype(np.int64).reshape(x.shape), step, lo


def order_of(d, is_key):
    """Dim of every 4-bit code of a row, in the order of the row's bytes (low half of a byte first)."""
    dims = np.empty(d, np.int64)
    m_all = d // 32
    if is_key:
        for c in range(4):
            for m in range(m_all):
                dims[8 * (c * m_all + m):][:8] = 32 * m + 8 * c + np.arange(8)
    else:
        for r in range(8):
            for m in range(m_all):
                dims[4 * (r * m_all + m):][:4] = 32 * m + 4 * r + np.arange(4)
    return dims


def int4_block(codes, step, lo, is_key):
    """Bytes of one block: codes [16, d], step, lo [16, groups]."""
    d, groups = codes.shape[1], step.shape[1]
    c = codes[:, order_of(d, is_key)]
    head = (c[:, 0::2] | (c[:, 1::2] << 4)).astype(np.uint8).reshape(-1)
    tail = np.empty((groups, 4, 2, 4), np.uint16)
    for r in range(16):
        for k, v in enumerate((step, lo)):
            tail[:, r % 4, k, r // 4] = (np.ascontiguousarray(v[r], np.float32).view(np.uint32) >> 16).astype(np.uint16)
    return np.concatenate([head, tail.reshape(-1).view(np.uint8)])


def int4_values(block, d, group, is_key):
    """(values [16, d] in 64 bits, steps [16, d]) of a block's bytes."""
    head = block[: 8 * d].reshape(16, d // 2)
    codes = np.empty((16, d), np.int64)
    codes[:, order_of(d, is_key)] = np.stack([head & 15, head >> 4], -1).reshape(16, d)
    tail = np.ascontiguousarray(block[8 * d:]).view(np.uint16).astype(np.uint32).reshape(d // group, 4, 2, 4)
    both = np.empty((16, d // group, 2))
    for r in range(16):
        both[r] = np.ascontiguousarray(tail[:, r % 4, :, r // 4] << 16).view(np.float32)
    step = np.repeat(both[..., 0], group, -1)
    return np.repeat(both[..., 1], group, -1) + step * codes, step


def rotate(x, pos, cos, sin, rotary, interleaved):
    """x [..., n, d], pos [n], in 64 bits."""
    x = x.astype(np.float64).copy()
    i = np.arange(rotary // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
    c, s = cos[pos].astype(np.float64), sin[pos].astype(np.float64)
    xa, xb = x[..., a], x[..., b]
    x[..., a], x[..., b] = xa * c - xb * s, xb * c + xa * s
    return x


def attend(q, K, V, scale, cap, lims):
    """q [n, d], K, V [rows, d], lims [n] in 64 bits -> out [n, d], lse [n], sum of weights times |v| [n, d], size of the logits [n]."""
    n, d = q.shape
    out, lse, mass, size = np.zeros((n, d)), np.full(n, NEG_INF), np.zeros((n, d)), np.zeros(n)
    for i in range(n):
        if lims[i] <= 0:
            continue
        s = (K[: lims[i]] @ q[i]) * scale
        size[i] = (np.abs(K[: lims[i]]) @ np.abs(q[i])).max() * scale
        if cap:
            s = cap * np.tanh(s / cap)
        top = s.max()
        w = np.exp(s - top)
        lse[i] = top + math.log(w.sum())
        w /= w.sum()
        out[i] = w @ V[: lims[i]]
        mass[i] = w @ np.abs(V[: lims[i]])
    return out, lse, mass, size


# ---- a cache on the device and what it stands for ------------------------------------------------------------------------------------

class Cache:
    """Pages full of stale bytes, a shuffled table, and the library's description of them."""

    def __init__(self, rng, batch, Hq, Hkv, d, fmt, page_rows, width, group=0, dtype="bf16", per_head=False, softcap=0.0, scale=0.0, spare=3):
        self.batch, self.Hq, self.Hkv, self.d, self.fmt, self.R, self.W, self.group = batch, Hq, Hkv, d, fmt, page_rows, width, group
        self.dtype, self.per_head, self.cap = dtype, per_head, softcap
        self.scale = scale or 1.0 / math.sqrt(d)
        self.t = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.n_pages = batch * width + spare
        self.desc = rk.make_paged(batch, Hq, Hkv, d, {"bf16": rk.PAGES_BF16, "f32": rk.PAGES_F32, "int4": rk.PAGES_INT4}[fmt], page_rows,
                                  self.n_pages, width, group, rk.BF16 if dtype == "bf16" else rk.F32, per_head, scale, softcap)
        self.block = 8 * d + 64 * (d // group) if fmt == "int4" else 16 * d * (2 if fmt == "bf16" else 4)
        shape = (self.n_pages, Hkv, page_rows // 16, self.block)
        # 0xFF bytes are NaN in every element type: nothing of a row that was not written may reach a result
        self.K, self.V = (torch.full(shape, 255, dtype=torch.uint8, device="cuda") for _ in range(2))
        self.table_np = rng.permutation(self.n_pages)[: batch * width].reshape(batch, width)
        self.table = torch.from_numpy(self.table_np.astype(np.int32)).cuda()

    def rows(self, pages, is_key, b, h, n):
        """(values [n, d] in 64 bits, steps or 0) of the first n rows."""
        host = pages.cpu().numpy()
        values, steps = np.empty((n, self.d)), np.zeros((n, self.d))
        for r0 in range(0, n, 16):
            block = host[self.table_np[b, r0 // self.R], h, r0 % self.R // 16]
            m = min(16, n - r0)
            if self.fmt == "int4":
                v, s = int4_values(block, self.d, self.group, is_key)
                steps[r0:r0 + m] = s[:m]
            elif self.fmt == "bf16":
                v = torch.from_numpy(block.copy()).view(torch.bfloat16).double().numpy().reshape(16, self.d)
            else:
                v = block.copy().view(np.float32).astype(np.float64).reshape(16, self.d)
            values[r0:r0 + m] = v[:m]
        return values, steps

    def fill(self, handle, rng, lengths, spread=1.0):
        """Rows 0 .. length of every sequence (and head), appended in one call."""
        most = int(np.max(lengths))
        K, V = (to_dev(rng.standard_normal((self.batch, self.Hkv, max(1, most), self.d)) * spread, self.t) for _ in range(2))
        per = np.asarray(lengths).reshape(self.batch, -1)
        for b in range(self.batch):      # one sequence at a time, since counts are one per sequence; heads beside it get no new rows
            for h in range(per.shape[1]):
                n = int(per[b, h])
                if n == 0:
                    continue
                heads = range(self.Hkv) if per.shape[1] == 1 else [h]
                one = rk.make_paged(1, self.Hq // self.Hkv * len(heads), len(heads), self.d, self.desc.page_format, self.R, self.n_pages, self.W,
                                    self.group, self.desc.dtype)
                if per.shape[1] == 1:
                    handle.paged_append(one, n, K[b:b + 1, :, :n], V[b:b + 1, :, :n], self.K, self.V, dev_i32([n]), self.table[b:b + 1])
                else:   # a single head's pages as a pool of their own
                    k, v = (p[:, h:h + 1].contiguous() for p in (self.K, self.V))
                    handle.paged_append(one, n, K[b:b + 1, h:h + 1, :n], V[b:b + 1, h:h + 1, :n], k, v, dev_i32([n]), self.table[b:b + 1])
                    self.K[:, h:h + 1], self.V[:, h:h + 1] = k, v
        torch.cuda.synchronize()
        assert handle.poll_status() == rk.RESTKV_OK


def dev_i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def to_dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().to(dtype)


def np64(t):
    return t.detach().double().cpu().numpy()


def tables(positions, rotary):
    angle = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(0, rotary, 2) / rotary)
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


@pytest.fixture(scope="module")
def handle():
    h = rk.Handle()
    yield h
    h.close()


# ---- appending ---------------------------------------------------------------------------------------------------------------------

# batch, query heads, KV heads, head_dim, page rows, rows before, tokens, rotary, interleaved
APPEND = [(1, 4, 1, 64, 16, 0, 1, 64, False), (2, 6, 3, 128, 32, 31, 1, 128, False), (3, 8, 2, 128, 64, 5, 70, 64, True), (2, 4, 4, 32, 16, 15, 18, 16, False),
          (1, 2, 2, 256, 48, 0, 130, 256, True), (2, 3, 1, 96, 16, 100, 9, 48, False), (1, 5, 5, 160, 128, 3, 40, 0, False), (4, 32, 8, 128, 64, 60, 300, 128, False)]


@pytest.mark.gpu
@pytest.mark.parametrize("spec", APPEND)
@pytest.mark.parametrize("fmt", ["bf16", "f32", "int4-bf16", "int4-f32"])
@pytest.mark.parametrize("strided", [False, True])
def test_append(handle, spec, fmt, strided):
    b, Hq, Hkv, d, R, before, t, rotary, interleaved = spec
    rng = np.random.default_rng(sum(spec[:8]) + len(fmt) + strided)
    dtype = "f32" if fmt.endswith("f32") else "bf16"
    fmt = fmt.split("-")[0]
    group = next(g for g in (64, 32) if d % g == 0) if t % 2 else max(g for g in (32, 64, 128) if d % g == 0)
    cache = Cache(rng, b, Hq, Hkv, d, fmt, R, -(-(before + t) // R) + 1, group if fmt == "int4" else 0, dtype)
    counts = np.array([max(0, t - 7 * i) for i in range(b)])
    lengths = before + counts
    if strided:
        fused = to_dev(rng.standard_normal((b, t, Hq + 2 * Hkv, d)), cache.t).transpose(1, 2)
        Q, K, V = fused.split([Hq, Hkv, Hkv], dim=1)
    else:
        Q, K, V = (to_dev(rng.standard_normal((b, H, t, d)), cache.t) for H in (Hq, Hkv, Hkv))
    P = before + t + 50
    positions = rng.integers(0, P, (b, t)).astype(np.int32)
    Q_out = torch.full((b, Hq, t, d), float("nan"), dtype=cache.t, device="cuda")
    kw = {}
    if rotary:
        cos, sin = tables(P, rotary)
        kw = {"rotation": rk.make_rotation(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), rotary, interleaved),
              "positions": dev_i32(positions)}
    stale_K, stale_V = cache.K.clone(), cache.V.clone()
    handle.paged_append(cache.desc, t, K, V, cache.K, cache.V, dev_i32(lengths), cache.table, counts=dev_i32(counts), Q=Q, Q_out=Q_out, **kw)
    torch.cuda.synchronize()
    assert handle.poll_status() == rk.RESTKV_OK

    # the queries: one rounding (8 significant bits: at most 2^-8) of an fp32 result whose own error is at most three roundings of its terms
    unit = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    for i in range(b):
        x = np64(Q[i])
        want = rotate(x, positions[i], cos, sin, rotary, interleaved) if rotary else x
        size = np.abs(x).max(-1, keepdims=True)
        got = np64(Q_out[i])
        assert np.all(got[:, counts[i]:] == 0)
        c = counts[i]
        if rotary:
            assert np.all(np.abs(got - want)[:, :c] <= unit * np.abs(want[:, :c]) + 2.0 ** -21 * size[:, :c])
        else:
            assert np.array_equal(got[:, :c], want[:, :c])
    # the rows, and nothing else
    touched_K, touched_V = torch.zeros_like(cache.K, dtype=torch.bool), torch.zeros_like(cache.V, dtype=torch.bool)
    for i in range(b):
        n = int(lengths[i])
        for h in range(Hkv):
            for is_key, pages, new, touched in ((True, cache.K, K, touched_K), (False, cache.V, V, touched_V)):
                x = np64(new[i, h])[: counts[i]]
                want = rotate(x, positions[i, : counts[i]], cos, sin, rotary, interleaved) if rotary and is_key else x
                size = np.abs(x).max(-1, keepdims=True) if len(x) else 0
                got, steps = (a[n - counts[i]:] for a in cache.rows(pages, is_key, i, h, n))
                if fmt != "int4":
                    if rotary and is_key:
                        assert np.all(np.abs(got - want) <= unit * np.abs(want) + 2.0 ** -21 * size)
                    else:
                        assert np.array_equal(got, want)
                else:
                    # nearest code: half a step, and the fp32 error of rotation, span and quotient
                    assert np.all(np.abs(got - want) <= 0.5 * steps + 2.0 ** -20 * size)
                    if not (rotary and is_key) and len(x):
                        codes, step, lo = quantise(x.astype(np.float32), group)
                        assert np.array_equal(got, np.repeat(lo.astype(np.float64), group, -1) + np.repeat(step.astype(np.float64), group, -1) * codes)
                for r in range(n - counts[i], n):
                    page, blk, q = cache.table_np[i, r // R], r % R // 16, r % 16
                    rb = cache.d // 2 if fmt == "int4" else cache.block // 16
                    touched[page, h, blk, q * rb:(q + 1) * rb] = True
                    if fmt == "int4":
                        for g in range(d // group):
                            for o in (0, 8):
                                at = 8 * d + 64 * g + 16 * (q % 4) + o + 2 * (q // 4)
                                touched[page, h, blk, at:at + 2] = True
    assert torch.equal(cache.K[~touched_K], stale_K[~touched_K])
    assert torch.equal(cache.V[~touched_V], stale_V[~touched_V])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,group", [(64, 32), (128, 64), (256, 128), (128, 128), (96, 32)])
def test_int4_block_bytes(handle, d, group, dtype):
    """A full block against the layout as the header states it, byte by byte, values on the grid's edges and far from it among them."""
    rng = np.random.default_rng(d + group)
    cache = Cache(rng, 1, 1, 1, d, "int4", 16, 1, group, dtype)
    x = rng.standard_normal((2, 16, d)).astype(np.float32)
    x[:, 1] = 0.0                                   # no span
    x[:, 2] = 3.25
    x[:, 3] = np.arange(d) % 16 - 7.0               # on the grid
    x[:, 4] = np.arange(d) % 31 * 0.5               # half-way between codes
    x[:, 5] += 100.0                                # far from 0
    x[:, 6] *= 1e-30
    x[:, 7] *= 1e30
    x[:, 8, :3] = [np.inf, -np.inf, np.nan]
    x[:, 9] = np.nan
    x[:, 10] = -5.0
    x[:, 11, 5] = 3e38
    x[:, 12] = -np.abs(x[:, 12])
    K, V = (to_dev(a[None, None], cache.t) for a in x)
    handle.paged_append(cache.desc, 16, K, V, cache.K, cache.V, dev_i32([16]), cache.table)
    torch.cuda.synchronize()
    page = int(cache.table_np[0, 0])
    for is_key, pages, new in ((True, cache.K, K), (False, cache.V, V)):
        codes, step, lo = quantise(new[0, 0].float().cpu().numpy(), group)
        assert np.array_equal(pages[page, 0, 0].cpu().numpy(), int4_block(codes, step, lo, is_key))


@pytest.mark.gpu
def test_append_positions_default_to_rows(handle):
    rng = np.random.default_rng(3)
    cache = Cache(rng, 2, 2, 2, 64, "bf16", 16, 4)
    cos, sin = tables(64, 64)
    rot = rk.make_rotation(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), 64)
    K, V = (to_dev(rng.standard_normal((2, 2, 6, 64)), torch.bfloat16) for _ in range(2))
    lengths = np.array([30, 17])
    handle.paged_append(cache.desc, 6, K, V, cache.K, cache.V, dev_i32(lengths), cache.table, rotation=rot)
    torch.cuda.synchronize()
    for b in range(2):
        for h in range(2):
            got = cache.rows(cache.K, True, b, h, int(lengths[b]))[0][lengths[b] - 6:]
            want = rotate(np64(K[b, h]), np.arange(lengths[b] - 6, lengths[b]), cos, sin, 64, False)
            assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -20)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_append_skips_what_has_no_place(handle, fmt):
    """Rows outside the table, table entries outside the pool and positions outside the tables: nothing is written, the status says so."""
    rng = np.random.default_rng(4)
    group = 32 if fmt == "int4" else 0
    K, V = (to_dev(rng.standard_normal((1, 1, 4, 64)), torch.bfloat16) for _ in range(2))
    cos, sin = tables(40, 64)
    rot = rk.make_rotation(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), 64)
    for kind in ("past the table", "before row 0", "page too large", "page negative", "position too large", "position negative"):
        cache = Cache(rng, 1, 1, 1, 64, fmt, 16, 2, group)
        stale = cache.K.clone(), cache.V.clone()
        length, kw = 20, {}
        if kind == "past the table":
            length = 36
        elif kind == "before row 0":
            length = 0
        elif kind.startswith("page"):
            cache.table[0, 1] = cache.n_pages if "large" in kind else -1
        else:
            kw = {"rotation": rot, "positions": dev_i32([[40 if "large" in kind else -1] * 4])}
        handle.paged_append(cache.desc, 4, K, V, cache.K, cache.V, dev_i32([length]), cache.table, **kw)
        assert handle.poll_status() == rk.ERR_INVALID_ARG, kind
        assert handle.poll_status() == rk.RESTKV_OK
        assert torch.equal(cache.K, stale[0]) and torch.equal(cache.V, stale[1]), kind


# ---- reading back ------------------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("spec", [(1, 1, 64, 16, [1], 32), (2, 2, 128, 32, [0, 77], 64), (3, 4, 128, 64, [130, 64, 1], 128), (1, 2, 256, 16, [40], 128),
                                  (2, 1, 96, 48, [50, 95], 32)])
@pytest.mark.parametrize("fmt", ["bf16", "f32", "int4-bf16", "int4-f32"])
def test_read(handle, spec, fmt):
    b, Hkv, d, R, lengths, group = spec
    rng = np.random.default_rng(b + d)
    dtype = "f32" if fmt.endswith("f32") else "bf16"
    fmt = fmt.split("-")[0]
    cache = Cache(rng, b, Hkv, Hkv, d, fmt, R, -(-max(lengths) // R) + 1, group if fmt == "int4" else 0, dtype)
    cache.fill(handle, rng, lengths)
    first = np.array([max(0, n // 2 - 3) for n in lengths])
    for start in (None, first):
        n_rows = max(lengths) + 3
        K, V = (torch.full((b, Hkv, n_rows, d), float("nan"), dtype=cache.t, device="cuda") for _ in range(2))
        handle.paged_read(cache.desc, cache.K, cache.V, dev_i32(lengths), cache.table, n_rows, K, V, first=None if start is None else dev_i32(start))
        torch.cuda.synchronize()
        for i in range(b):
            f = 0 if start is None else int(start[i])
            for h in range(Hkv):
                for got, pages, is_key in ((K, cache.K, True), (V, cache.V, False)):
                    want = cache.rows(pages, is_key, i, h, lengths[i])[0][f:]
                    m = len(want)
                    exact = want.astype(np.float32)      # offset + step * code has few bits: float32 rounds it once
                    exact = bf16_round(exact) if dtype == "bf16" else exact
                    assert np.array_equal(got[i, h, :m].float().cpu().numpy(), exact)
                    assert torch.all(got[i, h, m:] == 0)
    assert handle.poll_status() == rk.RESTKV_OK


# ---- attention -----------------------------------------------------------------------------------------------------------------------

def check_attention(handle, rng, cache, lengths, counts, t, q_scale=1.0, strided=False, note=""):
    b, Hq, Hkv, d = cache.batch, cache.Hq, cache.Hkv, cache.d
    G = Hq // Hkv
    q = rng.standard_normal((b, t, Hq, d) if strided else (b, Hq, t, d)) * q_scale
    Q = to_dev(q, cache.t)
    if strided:
        Q = Q.transpose(1, 2)
    out = torch.full((b, Hq, t, d), float("nan"), dtype=cache.t, device="cuda")
    lse = torch.full((b, Hq, t), float("nan"), device="cuda")
    ws = torch.empty(handle.paged_workspace_bytes(cache.desc, t), dtype=torch.uint8, device="cuda")
    ws.fill_(255)
    handle.paged_attend(cache.desc, t, Q, cache.K, cache.V, dev_i32(lengths), cache.table, out, ws, lse=lse,
                        counts=None if counts is None else dev_i32(counts))
    torch.cuda.synchronize()
    assert handle.poll_status() == rk.RESTKV_OK
    per = np.asarray(lengths).reshape(b, -1)
    got_o, got_l = np64(out), np64(lse)
    for i in range(b):
        c = t if counts is None else int(counts[i])
        for h in range(Hkv):
            n = int(per[i, h % per.shape[1]])
            K, _ = cache.rows(cache.K, True, i, h, n)
            V, steps = cache.rows(cache.V, False, i, h, n)
            lims = [n - (c - 1 - j) if j < c else 0 for j in range(t)]
            for g in range(G):
                hq = h * G + g
                qq = np64(Q[i, hq])
                o, l, mass, size = attend(qq, K, V, cache.scale, cache.cap, lims)
                empty = np.isneginf(l)
                assert np.array_equal(np.isneginf(got_l[i, hq]), empty), note
                assert np.all(got_o[i, hq][empty] == 0), note
                # a logit is an fp32 sum of d products (and in 4 bits of a scaled sum with an offset of 16 codes): at most
                # 2^-19 of the sum of their sizes; the cap adds its own rounding
                dl = 2.0 ** -19 * size + (2.0 ** -20 * cache.cap if cache.cap else 0.0) + 2.0 ** -20
                if cache.dtype == "f32":
                    bound = 2.0 ** -17 * mass + 4 * dl[:, None] * mass + 1e-30
                else:
                    # a weight (times the step, in 4 bits) is rounded to bf16 and meets codes of -8..7, V of the same size else;
                    # the output is rounded once
                    rest = steps.max(initial=0.0) * 8
                    bound = (2.0 ** -8 + 2.0 ** -15) * (mass + rest) + 4 * dl[:, None] * mass + 2.0 ** -8 * np.abs(o) + 1e-30
                err = np.abs(got_o[i, hq] - o)
                assert np.all(err <= bound), "%s: out %.3f of the bound" % (note, float((err / bound).max()))
                ok = ~empty
                assert np.all(np.abs(got_l[i, hq][ok] - l[ok]) <= (2 * dl + 2.0 ** -21 * np.abs(l) + 2.0 ** -18)[ok]), note


# batch, query heads, KV heads, head_dim, page rows, lengths
DECODE = [(1, 4, 1, 128, 16, [1]), (2, 8, 2, 128, 32, [15, 16]), (3, 8, 2, 64, 16, [17, 0, 260]), (1, 32, 8, 128, 64, [1000]), (4, 8, 8, 128, 16, [1, 33, 2048, 700]),
          (2, 16, 1, 128, 64, [129, 500]), (1, 24, 1, 128, 16, [300]), (2, 6, 2, 64, 48, [100, 47]), (1, 2, 1, 256, 32, [333]), (2, 5, 5, 96, 16, [64, 31]),
          (1, 7, 1, 32, 16, [90]), (1, 40, 1, 64, 16, [70]), (9, 8, 4, 128, 16, [5, 1, 0, 16, 400, 3, 31, 32, 33])]


@pytest.mark.gpu
@pytest.mark.parametrize("spec", DECODE)
@pytest.mark.parametrize("fmt", ["bf16", "f32", "int4-bf16", "int4-f32"])
@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_attend_one_token(handle, spec, fmt, cap):
    b, Hq, Hkv, d, R, lengths = spec
    rng = np.random.default_rng(Hq + d + len(fmt))
    dtype = "f32" if fmt.endswith("f32") else "bf16"
    fmt = fmt.split("-")[0]
    for group in [g for g in (32, 64, 128) if d % g == 0] if fmt == "int4" else [0]:
        cache = Cache(rng, b, Hq, Hkv, d, fmt, R, -(-max(lengths) // R) + 1, group, dtype, softcap=cap)
        cache.fill(handle, rng, lengths)
        check_attention(handle, rng, cache, lengths, None, 1, q_scale=2.0, note="group %d" % group)


# batch, query heads, KV heads, head_dim, page rows, lengths, counts, tokens
CHUNK = [(1, 4, 1, 128, 16, [2], None, 2), (2, 8, 2, 128, 32, [20, 37], [3, 5], 5), (1, 8, 2, 128, 64, [200], None, 33), (2, 4, 4, 64, 16, [70, 3], [64, 3], 64),
         (3, 6, 2, 128, 16, [5, 100, 0], [7, 20, 0], 20), (1, 32, 8, 128, 64, [400], None, 150), (1, 2, 1, 256, 16, [90], None, 40), (2, 3, 1, 96, 16, [40, 20], [9, 2], 9),
         (1, 16, 1, 128, 16, [300], None, 130), (1, 1, 1, 64, 16, [500], None, 300), (1, 20, 1, 128, 32, [150], None, 17), (2, 4, 1, 128, 16, [257, 129], [129, 129], 129)]


@pytest.mark.gpu
@pytest.mark.parametrize("spec", CHUNK)
@pytest.mark.parametrize("fmt", ["bf16", "f32", "int4-bf16", "int4-f32"])
@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_attend_several_tokens(handle, spec, fmt, cap):
    b, Hq, Hkv, d, R, lengths, counts, t = spec
    rng = np.random.default_rng(Hq + d + t)
    dtype = "f32" if fmt.endswith("f32") else "bf16"
    fmt = fmt.split("-")[0]
    for group in [g for g in (32, 64, 128) if d % g == 0] if fmt == "int4" else [0]:
        cache = Cache(rng, b, Hq, Hkv, d, fmt, R, -(-max(lengths) // R), group, dtype, softcap=cap)
        cache.fill(handle, rng, lengths)
        check_attention(handle, rng, cache, lengths, counts, t, q_scale=1.5, strided=True, note="group %d" % group)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("t", [1, 3, 40])
def test_attend_lengths_per_head(handle, fmt, t):
    rng = np.random.default_rng(5)
    cache = Cache(rng, 2, 8, 4, 128, fmt, 16, 20, 64 if fmt == "int4" else 0, per_head=True)
    lengths = np.array([[1, 300, 64, 17], [0, 5, 200, 33]])
    cache.fill(handle, rng, lengths)
    check_attention(handle, rng, cache, lengths, None, t)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("t", [1, 2, 50])
@pytest.mark.parametrize("q_scale", [0.0, 40.0, 1000.0])
def test_attend_extreme_logits(handle, fmt, t, q_scale):
    """Uniform weights, and weights of which one carries everything."""
    rng = np.random.default_rng(6)
    cache = Cache(rng, 1, 8, 2, 128, fmt, 32, 10, 64 if fmt == "int4" else 0)
    cache.fill(handle, rng, [310])
    check_attention(handle, rng, cache, [310], None, t, q_scale=q_scale)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("spec", [(1, 32, 8, 1, 20000), (8, 32, 8, 1, 3000), (1, 32, 8, 600, 5000), (16, 16, 16, 4, 500)])
def test_attend_is_deterministic(handle, fmt, spec):
    b, Hq, Hkv, t, n = spec
    rng = np.random.default_rng(7)
    cache = Cache(rng, b, Hq, Hkv, 128, fmt, 64, -(-n // 64), 64 if fmt == "int4" else 0)
    lengths = [max(0, n - 37 * i) for i in range(b)]
    cache.fill(handle, rng, lengths)
    Q = to_dev(rng.standard_normal((b, Hq, t, 128)), torch.bfloat16)
    ws = torch.empty(handle.paged_workspace_bytes(cache.desc, t), dtype=torch.uint8, device="cuda")
    results = []
    for _ in range(3):
        out, lse = torch.empty_like(Q), torch.empty(b, Hq, t, device="cuda")
        handle.paged_attend(cache.desc, t, Q, cache.K, cache.V, dev_i32(lengths), cache.table, out, ws, lse=lse)
        results.append((out, lse))
        ws.fill_(255)
    torch.cuda.synchronize()
    for out, lse in results[1:]:
        assert torch.equal(out, results[0][0]) and torch.equal(lse, results[0][1])


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("t", [1, 50])
def test_attend_and_read_report_bad_tables(handle, fmt, t):
    """A page number outside the pool hides that page's rows, a length past the table counts as the table's; the status says so."""
    rng = np.random.default_rng(8)
    cache = Cache(rng, 1, 4, 1, 128, fmt, 16, 6, 32 if fmt == "int4" else 0)
    cache.fill(handle, rng, [96])
    Q = to_dev(rng.standard_normal((1, 4, t, 128)), torch.bfloat16)
    ws = torch.empty(handle.paged_workspace_bytes(cache.desc, t), dtype=torch.uint8, device="cuda")
    want, out = torch.empty_like(Q), torch.empty_like(Q)
    K, V = (torch.empty(1, 1, 100, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    handle.paged_attend(cache.desc, t, Q, cache.K, cache.V, dev_i32([96]), cache.table, want, ws)
    assert handle.poll_status() == rk.RESTKV_OK
    handle.paged_attend(cache.desc, t, Q, cache.K, cache.V, dev_i32([97]), cache.table, out, ws)
    assert handle.poll_status() == rk.ERR_INVALID_ARG
    assert torch.equal(out, want)
    handle.paged_attend(cache.desc, t, Q, cache.K, cache.V, dev_i32([-5]), cache.table, out, ws)
    assert handle.poll_status() == rk.RESTKV_OK
    assert torch.all(out == 0)
    for bad in (cache.n_pages, -1, 2 ** 31 - 1):
        table = cache.table.clone()
        table[0, 2] = bad
        handle.paged_attend(cache.desc, t, Q, cache.K, cache.V, dev_i32([96]), table, out, ws)
        assert handle.poll_status() == rk.ERR_INVALID_ARG
        assert bool(torch.isfinite(out.float()).all())
        handle.paged_read(cache.desc, cache.K, cache.V, dev_i32([96]), table, 100, K, V)
        assert handle.poll_status() == rk.ERR_INVALID_ARG
        assert torch.all(K[0, 0, 32:48] == 0) and torch.all(V[0, 0, 32:48] == 0) and torch.all(K[0, 0, 96:] == 0)
        assert bool((K[0, 0, :32] != 0).any()) and bool((K[0, 0, 48:96] != 0).any())


@pytest.mark.gpu
def test_attend_on_another_stream_and_in_a_graph(handle):
    rng = np.random.default_rng(9)
    cache = Cache(rng, 2, 8, 2, 128, "int4", 32, 20, 64)
    cache.fill(handle, rng, [600, 333])
    Q = to_dev(rng.standard_normal((2, 8, 1, 128)), torch.bfloat16)
    lengths = dev_i32([600, 333])
    ws = torch.empty(handle.paged_workspace_bytes(cache.desc, 1), dtype=torch.uint8, device="cuda")
    want, out = torch.empty_like(Q), torch.zeros_like(Q)
    handle.paged_attend(cache.desc, 1, Q, cache.K, cache.V, lengths, cache.table, want, ws)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    handle.paged_attend(cache.desc, 1, Q, cache.K, cache.V, lengths, cache.table, out, ws, stream=stream)
    stream.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        handle.paged_attend(cache.desc, 1, Q, cache.K, cache.V, lengths, cache.table, out, ws)
    lengths.copy_(dev_i32([601, 100]))      # rows that the graph did not know of; the 601st is stale: take one fewer
    lengths.copy_(dev_i32([590, 100]))
    graph.replay()
    handle.paged_attend(cache.desc, 1, Q, cache.K, cache.V, lengths, cache.table, want, ws)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.gpu
def test_offsets_past_32_bits(handle):
    """Pages of more than 2^32 bytes: rows of the last page are written, seen and read where they are."""
    d, R, Hkv = 128, 256, 8
    page_bytes = Hkv * R * d * 2
    n_pages = (1 << 32) // page_bytes + 3
    K, V = (torch.empty(n_pages, Hkv, R, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    desc = rk.make_paged(1, 8, Hkv, d, rk.PAGES_BF16, R, n_pages, 2)
    table = dev_i32([[n_pages - 1, n_pages - 2]])
    g = torch.Generator("cuda").manual_seed(1)
    new_K, new_V = (torch.randn(1, Hkv, 300, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    handle.paged_append(desc, 300, new_K, new_V, K, V, dev_i32([300]), table)
    back_K, back_V = torch.empty_like(new_K), torch.empty_like(new_V)
    handle.paged_read(desc, K, V, dev_i32([300]), table, 300, back_K, back_V)
    assert torch.equal(back_K, new_K) and torch.equal(back_V, new_V)
    assert torch.equal(K[n_pages - 1], new_K[0, :, :256]) and torch.equal(V[n_pages - 2, :, :44], new_V[0, :, 256:])
    Q = torch.randn(1, 8, 1, d, generator=g, device="cuda").to(torch.bfloat16)
    out = torch.empty_like(Q)
    ws = torch.empty(handle.paged_workspace_bytes(desc, 1), dtype=torch.uint8, device="cuda")
    handle.paged_attend(desc, 1, Q, K, V, dev_i32([300]), table, out, ws)
    w = torch.softmax((Q.double() @ new_K.double().transpose(-1, -2)) / math.sqrt(d), -1)
    want = w @ new_V.double()
    # weights rounded to bf16, the output rounded to bf16
    assert torch.all((out.double() - want).abs() <= 2.0 ** -8 * (w @ new_V.double().abs()) + 2.0 ** -8 * want.abs() + 1e-4)


# ---- refusals -------------------------------------------------------------------------------------------------------------------------

def good(**kw):
    a = dict(batch=1, n_q_heads=8, n_kv_heads=2, head_dim=128, page_format=rk.PAGES_INT4, page_rows=64, n_pages=10, table_width=4, group=64)
    a.update(kw)
    return rk.make_paged(**a)


REFUSED = [(dict(batch=0), rk.ERR_INVALID_ARG), (dict(n_q_heads=7), rk.ERR_INVALID_ARG), (dict(n_kv_heads=0), rk.ERR_INVALID_ARG), (dict(page_rows=24), rk.ERR_INVALID_ARG),
           (dict(page_rows=0), rk.ERR_INVALID_ARG), (dict(n_pages=0), rk.ERR_INVALID_ARG), (dict(table_width=0), rk.ERR_INVALID_ARG), (dict(group=48), rk.ERR_INVALID_ARG),
           (dict(group=0), rk.ERR_INVALID_ARG), (dict(head_dim=64, group=128), rk.ERR_INVALID_ARG), (dict(page_format=3), rk.ERR_INVALID_ARG), (dict(dtype=7), rk.ERR_INVALID_ARG),
           (dict(softcap=-1.0), rk.ERR_INVALID_ARG), (dict(softcap=float("nan")), rk.ERR_INVALID_ARG), (dict(softmax_scale=-1.0), rk.ERR_INVALID_ARG), (dict(lengths_per_head=2), rk.ERR_INVALID_ARG),
           (dict(head_dim=80), rk.ERR_UNSUPPORTED), (dict(head_dim=288, group=32), rk.ERR_UNSUPPORTED), (dict(page_format=rk.PAGES_F32), rk.ERR_UNSUPPORTED),
           (dict(page_format=rk.PAGES_BF16, dtype=rk.F32), rk.ERR_UNSUPPORTED), (dict(table_width=2 ** 26), rk.ERR_UNSUPPORTED), (dict(batch=70000), rk.ERR_UNSUPPORTED)]


@pytest.mark.parametrize("change,status", REFUSED)
def test_sizes_of_refused_caches_are_zero(change, status):
    lib = rk.load_library()
    assert lib.restkv_paged_page_bytes(ctypes.byref(good(**change))) == 0
    assert lib.restkv_paged_workspace_bytes(ctypes.byref(good(**change)), 1) == 0


def test_page_bytes():
    lib = rk.load_library()
    for kw, want in ((dict(), 2 * 64 * (64 + 8)), (dict(group=32), 2 * 64 * (64 + 16)), (dict(page_format=rk.PAGES_BF16, group=0), 2 * 64 * 256),
                     (dict(page_format=rk.PAGES_F32, dtype=rk.F32), 2 * 64 * 512), (dict(head_dim=96, group=32, page_rows=16), 2 * 16 * (48 + 12))):
        assert lib.restkv_paged_page_bytes(ctypes.byref(good(**kw))) == want
    assert lib.restkv_paged_page_bytes(None) == 0
    assert lib.restkv_paged_workspace_bytes(ctypes.byref(good()), 0) == 0
    assert lib.restkv_paged_workspace_bytes(ctypes.byref(good()), 1) > 0


def test_null_handle_is_rejected():
    lib = rk.load_library()
    c = good()
    assert lib.restkv_paged_append(None, ctypes.byref(c), 1, None, None, None, None, None, None, None, None, None, None, None, None) == rk.ERR_INVALID_ARG
    assert lib.restkv_paged_attend(None, ctypes.byref(c), 1, None, None, None, None, None, None, None, None, None, 0, None) == rk.ERR_INVALID_ARG
    assert lib.restkv_paged_read(None, ctypes.byref(c), None, None, None, None, None, 1, None, None, None) == rk.ERR_INVALID_ARG


def test_rows_and_rotation_helpers_refuse_what_they_cannot_describe():
    x = torch.zeros(1, 2, 3, 8)
    assert (rk.make_rows(x).stride_b, rk.make_rows(x).stride_h, rk.make_rows(x).stride_n) == (48, 24, 8)
    with pytest.raises(ValueError):
        rk.make_rows(x[0])
    with pytest.raises(ValueError):
        rk.make_rows(x.transpose(2, 3))
    with pytest.raises(ValueError):
        rk.make_rows(torch.zeros(8).expand(2, 2, 3, 8))
    with pytest.raises(ValueError):
        rk.make_rotation(torch.zeros(4, 8), torch.zeros(4, 7), 16)
    with pytest.raises(ValueError):
        rk.make_rotation(torch.zeros(4, 8, dtype=torch.float64), torch.zeros(4, 8, dtype=torch.float64), 16)


@pytest.mark.gpu
def test_refusals_enqueue_nothing(handle):
    rng = np.random.default_rng(10)
    cache = Cache(rng, 1, 8, 2, 128, "int4", 64, 4, 64)
    stale = cache.K.clone()
    Q = to_dev(rng.standard_normal((1, 8, 2, 128)), torch.bfloat16)
    K, V = (to_dev(rng.standard_normal((1, 2, 2, 128)), torch.bfloat16) for _ in range(2))
    out = torch.full_like(Q, 7.0)
    n = dev_i32([100])
    ws = torch.empty(handle.paged_workspace_bytes(cache.desc, 2), dtype=torch.uint8, device="cuda")
    cos, sin = (torch.zeros(200, 64, device="cuda") for _ in range(2))
    rot = rk.make_rotation(cos, sin, 128)
    launches = handle.launch_count()

    def status(call, *a, **k):
        with pytest.raises(rk.RestKVError) as e:
            call(*a, **k)
        return e.value.status

    for change, want in REFUSED:
        bad = good(**change)
        assert status(handle.paged_append, bad, 2, K, V, cache.K, cache.V, n, cache.table) == want, change
        assert status(handle.paged_attend, bad, 2, Q, cache.K, cache.V, n, cache.table, out, ws) == want, change
        assert status(handle.paged_read, bad, cache.K, cache.V, n, cache.table, 2, K, V) == want, change
    ok = cache.desc
    assert status(handle.paged_append, ok, 0, K, V, cache.K, cache.V, n, cache.table) == rk.ERR_INVALID_ARG
    assert status(handle.paged_append, ok, 2, K, V, cache.K, cache.V, n, cache.table, Q=Q) == rk.ERR_INVALID_ARG
    assert status(handle.paged_append, ok, 2, K, V, cache.K, cache.V, None, cache.table) == rk.ERR_INVALID_ARG
    assert status(handle.paged_append, ok, 2, K.view(-1)[4:260].view(1, 1, 2, 128), V, cache.K, cache.V, n, cache.table) == rk.ERR_INVALID_ARG      # 8 bytes off
    odd = torch.zeros(1, 2, 2, 132, dtype=torch.bfloat16, device="cuda")[..., :128]
    assert status(handle.paged_append, ok, 2, odd, V, cache.K, cache.V, n, cache.table) == rk.ERR_INVALID_ARG
    for wrong in (dict(rotary_dim=24), dict(rotary_dim=0), dict(rotary_dim=144), dict(interleaved=2), dict(n_positions=0), dict(cos=None)):
        r = rk.Rotation(rot.cos, rot.sin, 200, 128, 0)
        for k, v in wrong.items():
            setattr(r, k, v)
        assert status(handle.paged_append, ok, 2, K, V, cache.K, cache.V, n, cache.table, rotation=r) == rk.ERR_INVALID_ARG, wrong
    per_head = good(page_rows=64, n_pages=cache.n_pages, lengths_per_head=1)
    assert status(handle.paged_append, per_head, 2, K, V, cache.K, cache.V, dev_i32([[100, 100]]), cache.table, rotation=rot) == rk.ERR_INVALID_ARG
    assert status(handle.paged_attend, ok, 0, Q, cache.K, cache.V, n, cache.table, out, ws) == rk.ERR_INVALID_ARG
    assert status(handle.paged_attend, ok, 2, Q, cache.K, cache.V, n, None, out, ws) == rk.ERR_INVALID_ARG
    assert status(handle.paged_attend, ok, 2, Q, cache.K, cache.V, n, cache.table, out, ws[: ws.numel() - 256]) == rk.ERR_WORKSPACE
    assert status(handle.paged_attend, ok, 2, Q, cache.K, cache.V, n, cache.table, out, ws[16:]) == rk.ERR_WORKSPACE
    assert status(handle.paged_read, ok, cache.K, cache.V, n, cache.table, 0, K, V) == rk.ERR_INVALID_ARG
    assert status(handle.paged_read, ok, cache.K, cache.V, n, cache.table, 2, None, V) == rk.ERR_INVALID_ARG
    assert handle.launch_count() == launches
    torch.cuda.synchronize()
    assert torch.equal(cache.K, stale) and torch.all(out == 7.0)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("per_head", [False, True])
def test_attend_many_sequences(handle, fmt, per_head):
    """More units of work than the device keeps counters for, and than it has SMs; lengths that share no pattern."""
    rng = np.random.default_rng(11)
    b, Hkv = 90, 3
    cache = Cache(rng, b, 2 * Hkv, Hkv, 64, fmt, 16, 12, 32 if fmt == "int4" else 0, per_head=per_head)
    lengths = rng.integers(0, 190, (b, Hkv) if per_head else (b,))
    lengths.flat[3] = 0
    lengths.flat[5] = 192
    cache.fill(handle, rng, lengths)
    check_attention(handle, rng, cache, lengths, None, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("steps", [2.0 ** -30, 2.0 ** -12, 2.0 ** 12, 2.0 ** 40])
@pytest.mark.parametrize("t", [1, 40])
def test_attend_values_of_any_size(handle, fmt, steps, t):
    """V far from 1, and in one cache rows that are 2^20 times larger than the rest, which carry little weight or all of it."""
    rng = np.random.default_rng(12)
    cache = Cache(rng, 1, 4, 1, 128, fmt, 16, 40, 64 if fmt == "int4" else 0)
    K = rng.standard_normal((1, 1, 600, 128))
    V = rng.standard_normal((1, 1, 600, 128)) * steps
    V[:, :, 17::100] *= 2.0 ** 20
    V[:, :, 400:432] = 0.0
    handle.paged_append(cache.desc, 600, to_dev(K, cache.t), to_dev(V, cache.t), cache.K, cache.V, dev_i32([600]), cache.table)
    check_attention(handle, rng, cache, [600], None, t, q_scale=3.0)


# Calls of many query rows: enough of them (64 of a KV head, 1536 together) that they go by tiles of 128 against tiles of 128 cache rows.
IN_CHUNKS = [(2, 4, 4, 64, 16, [270, 3], [200, 3], 200), (1, 8, 2, 64, 32, [700], None, 256), (3, 6, 2, 128, 16, [130, 100, 0], [120, 20, 0], 120),
             (1, 1, 1, 64, 16, [1700], None, 1600), (1, 12, 4, 128, 48, [129], None, 129), (4, 8, 1, 128, 16, [64, 65, 191, 48], [48, 1, 48, 48], 48)]


@pytest.mark.gpu
@pytest.mark.parametrize("spec", IN_CHUNKS)
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_attend_in_chunks(handle, spec, fmt, cap):
    b, Hq, Hkv, d, R, lengths, counts, t = spec
    rng = np.random.default_rng(Hq + d + t)
    for group in [g for g in (32, 64, 128) if d % g == 0] if fmt == "int4" else [0]:
        cache = Cache(rng, b, Hq, Hkv, d, fmt, R, -(-max(lengths) // R), group, softcap=cap)
        cache.fill(handle, rng, lengths)
        check_attention(handle, rng, cache, lengths, counts, t, q_scale=1.5, strided=True, note="group %d" % group)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_attend_in_chunks_lengths_per_head(handle, fmt):
    rng = np.random.default_rng(13)
    cache = Cache(rng, 2, 8, 4, 128, fmt, 16, 20, 64 if fmt == "int4" else 0, per_head=True)
    lengths = np.array([[1, 300, 64, 117], [0, 105, 200, 133]])
    cache.fill(handle, rng, lengths)
    check_attention(handle, rng, cache, lengths, None, 100)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("q_scale", [0.0, 40.0, 1000.0])
def test_attend_in_chunks_extreme_logits(handle, fmt, cap, q_scale):
    rng = np.random.default_rng(14)
    cache = Cache(rng, 1, 8, 2, 128, fmt, 32, 10, 64 if fmt == "int4" else 0, softcap=cap)
    cache.fill(handle, rng, [310])
    check_attention(handle, rng, cache, [310], None, 200, q_scale=q_scale)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("t", [1, 3, 400])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_logits_that_grow(handle, fmt, t, d):
    """Every row's key is longer than the one before it, in every dim alike, so that what a row's weights refer to is left behind again
    and again: by rows with steps of one sign, and with a jump inside a tile."""
    rng = np.random.default_rng(15)
    cache = Cache(rng, 1, 4, 1, d, fmt, 16, 45, 32 if fmt == "int4" else 0)
    n = 700
    K = np.linspace(0.0, 6.0, n)[None, None, :, None] * np.sign(rng.standard_normal((1, 1, 1, d))) + 0.1 * rng.standard_normal((1, 1, n, d))
    K[:, :, 333:] *= 2.0
    V = rng.standard_normal((1, 1, n, d))
    handle.paged_append(cache.desc, n, to_dev(K, cache.t), to_dev(V, cache.t), cache.K, cache.V, dev_i32([n]), cache.table)
    check_attention(handle, rng, cache, [n], None, t, q_scale=4.0)


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [2.0 ** -30, 2.0 ** -12, 2.0 ** 12, 2.0 ** 40])
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_attend_in_chunks_values_of_any_size(handle, fmt, steps):
    rng = np.random.default_rng(16)
    cache = Cache(rng, 1, 4, 1, 128, fmt, 16, 40, 64 if fmt == "int4" else 0)
    K = rng.standard_normal((1, 1, 600, 128))
    V = rng.standard_normal((1, 1, 600, 128)) * steps
    V[:, :, 17::100] *= 2.0 ** 20
    V[:, :, 400:432] = 0.0
    handle.paged_append(cache.desc, 600, to_dev(K, cache.t), to_dev(V, cache.t), cache.K, cache.V, dev_i32([600]), cache.table)
    check_attention(handle, rng, cache, [600], None, 400, q_scale=3.0)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_attend_in_chunks_reports_bad_tables(handle, fmt):
    rng = np.random.default_rng(17)
    cache = Cache(rng, 1, 4, 1, 128, fmt, 16, 32, 32 if fmt == "int4" else 0)
    cache.fill(handle, rng, [512])
    Q = to_dev(rng.standard_normal((1, 4, 400, 128)), torch.bfloat16)
    ws = torch.empty(handle.paged_workspace_bytes(cache.desc, 400), dtype=torch.uint8, device="cuda")
    want, out = torch.empty_like(Q), torch.empty_like(Q)
    handle.paged_attend(cache.desc, 400, Q, cache.K, cache.V, dev_i32([512]), cache.table, want, ws)
    assert handle.poll_status() == rk.RESTKV_OK
    handle.paged_attend(cache.desc, 400, Q, cache.K, cache.V, dev_i32([513]), cache.table, out, ws)
    assert handle.poll_status() == rk.ERR_INVALID_ARG
    assert torch.equal(out, want)
    for bad in (cache.n_pages, -1, 2 ** 31 - 1):
        table = cache.table.clone()
        table[0, 9] = bad
        handle.paged_attend(cache.desc, 400, Q, cache.K, cache.V, dev_i32([500]), table, out, ws)
        assert handle.poll_status() == rk.ERR_INVALID_ARG
        assert bool(torch.isfinite(out.float()).all())


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_attend_chunk_equals_its_tokens(handle, fmt):
    """A chunk over a cache, and its tokens one call at a time with the lengths that they see, by the two kernels: both within a rounding
    of the output and of the weights of the exact result."""
    rng = np.random.default_rng(18)
    cache = Cache(rng, 2, 8, 2, 128, fmt, 32, 12, 64 if fmt == "int4" else 0)
    lengths, t = [380, 210], 128
    cache.fill(handle, rng, lengths)
    Q = to_dev(rng.standard_normal((2, 8, t, 128)), torch.bfloat16)
    ws = torch.empty(handle.paged_workspace_bytes(cache.desc, t), dtype=torch.uint8, device="cuda")
    whole, lse = torch.empty_like(Q), torch.empty(2, 8, t, device="cuda")
    handle.paged_attend(cache.desc, t, Q, cache.K, cache.V, dev_i32(lengths), cache.table, whole, ws, lse=lse)
    ws1 = torch.empty(handle.paged_workspace_bytes(cache.desc, 1), dtype=torch.uint8, device="cuda")
    for i in (0, 1, 63, 64, 127):
        one, l1 = torch.empty(2, 8, 1, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 8, 1, device="cuda")
        handle.paged_attend(cache.desc, 1, Q[:, :, i:i + 1].contiguous(), cache.K, cache.V, dev_i32([n - (t - 1 - i) for n in lengths]), cache.table, one,
                            ws1, lse=l1)
        torch.cuda.synchronize()
        # values are at most 5 or so, and a weighted mean of them no larger: two roundings of weights and one of each output
        assert float((one[:, :, 0].float() - whole[:, :, i].float()).abs().max()) <= 5.5 * (2 * 2.0 ** -8 + 2 * 2.0 ** -8)
        assert float((l1[:, :, 0] - lse[:, :, i]).abs().max()) <= 2.0 ** -12
    assert handle.poll_status() == rk.RESTKV_OK


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "f32", "int4-bf16", "int4-f32"])
@pytest.mark.parametrize("spec", [(2, 8, 2, 128, 16, [300, 277], 200), (1, 3, 1, 96, 16, [40], 40), (1, 4, 4, 64, 32, [513], 400), (3, 8, 2, 128, 48, [7, 1, 100], 1),
                                  (2, 4, 1, 256, 16, [33, 18], 17)])
def test_no_paged_write_lands_outside_a_buffer(handle, fmt, spec):
    """Pages, outputs and workspace out of one allocation with 4 KB bands of a pattern between them, which are intact afterwards."""
    b, Hq, Hkv, d, R, lengths, t = spec
    rng = np.random.default_rng(19)
    dtype = "f32" if fmt.endswith("f32") else "bf16"
    cache = Cache(rng, b, Hq, Hkv, d, fmt.split("-")[0], R, -(-max(lengths) // R), 32 if fmt.startswith("int4") else 0, dtype)
    size = 4 if dtype == "f32" else 2
    parts = {"K": cache.K.numel(), "V": cache.V.numel(), "q": b * Hq * t * d * size, "out": b * Hq * t * d * size, "lse": b * Hq * t * 4,
             "ws": handle.paged_workspace_bytes(cache.desc, t), "Kr": b * Hkv * max(lengths) * d * size, "Vr": b * Hkv * max(lengths) * d * size}
    at, total = {}, 4096
    for k, n in parts.items():
        at[k] = total
        total = -(-(total + n) // 256) * 256 + 4096
    memory = torch.full((total,), 0xA5, dtype=torch.uint8, device="cuda")
    part = {k: memory[at[k]: at[k] + n] for k, n in parts.items()}
    inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    for k, n in parts.items():
        inside[at[k]: at[k] + n] = True
    new, Q = to_dev(rng.standard_normal((2, b, Hkv, max(lengths), d)), cache.t), to_dev(rng.standard_normal((b, Hq, t, d)), cache.t)
    angles = torch.arange(max(lengths), device="cuda")[:, None] * torch.linspace(1.0, 0.01, d // 2, device="cuda")
    rotation = rk.make_rotation(angles.cos().contiguous(), angles.sin().contiguous(), d)
    n, most = dev_i32(lengths), max(lengths)
    # the sequences but for the last t rows, then those with their queries, attention, and all of it read back
    handle.paged_append(cache.desc, most, new[0], new[1], part["K"], part["V"], n, cache.table, counts=n)
    handle.paged_append(cache.desc, t, new[0, :, :, -t:], new[1, :, :, -t:], part["K"], part["V"], n, cache.table, counts=dev_i32([min(t, x) for x in lengths]),
                        rotation=rotation, Q=Q, Q_out=part["q"])
    out = part["q"].view(cache.t).view(b, Hq, t, d)
    handle.paged_attend(cache.desc, t, out, part["K"], part["V"], n, cache.table, part["out"], part["ws"], lse=part["lse"].view(torch.float32),
                        counts=dev_i32([min(t, x) for x in lengths]))
    handle.paged_read(cache.desc, part["K"], part["V"], n, cache.table, most, part["Kr"], part["Vr"])
    torch.cuda.synchronize()
    assert handle.poll_status() == rk.RESTKV_OK
    assert bool((memory[~inside] == 0xA5).all())
    # and everything that is promised has been written
    assert bool(torch.isfinite(part["out"].view(cache.t).float()).all())
    assert bool(torch.isfinite(part["Kr"].view(cache.t).float()).all()) and bool(torch.isfinite(part["Vr"].view(cache.t).float()).all())
    pages = part["K"].view_as(cache.K)
    spare = torch.ones(cache.n_pages, dtype=torch.bool)
    spare[torch.from_numpy(cache.table_np.reshape(-1))] = False
    assert bool((pages[spare.cuda()] == 0xA5).all())


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("t", [1, 6, 200])
def test_attend_in_fp32_throughout(handle, fmt, t):
    """Kernel path 1: the same call within the bounds of the tensor cores', and within those of fp32 sums and one rounding of the output."""
    rng = np.random.default_rng(20)
    cache = Cache(rng, 2, 8, 2, 128, fmt, 16, 20, 64 if fmt == "int4" else 0, softcap=8.0)
    cache.fill(handle, rng, [310, 205])
    handle.set_kernel_path(1)
    try:
        check_attention(handle, rng, cache, [310, 205], None, t)
    finally:
        handle.set_kernel_path(0)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "f32", "int4-bf16", "int4-f32"])
@pytest.mark.parametrize("page_rows", [16, 48])
@pytest.mark.parametrize("per_head", [False, True])
def test_read_from_before_the_first_row(handle, fmt, page_rows, per_head):
    """Any first row, negative ones among them, in calls small enough for a block of 16 rows per warp and large enough for runs of blocks."""
    b, Hkv, d = 5, 8, 64
    rng = np.random.default_rng(21)
    dtype = "f32" if fmt.endswith("f32") else "bf16"
    fmt = fmt.split("-")[0]
    cache = Cache(rng, b, Hkv, Hkv, d, fmt, page_rows, -(-560 // page_rows), 32 if fmt == "int4" else 0, dtype, per_head=per_head)
    lengths = np.array([540, 37, 0, 512, 301])
    if per_head:
        lengths = np.maximum(lengths[:, None] - 13 * np.arange(Hkv), 0)
    cache.fill(handle, rng, lengths)
    per = np.broadcast_to(lengths.reshape(b, -1), (b, Hkv))
    host = {}
    for is_key, pages in ((True, cache.K), (False, cache.V)):
        for i in range(b):
            for h in range(Hkv):
                x = cache.rows(pages, is_key, i, h, int(per[i, h]))[0].astype(np.float32)
                host[is_key, i, h] = bf16_round(x) if dtype == "bf16" else x
    runs_of_blocks = 16 * (-(-32 * torch.cuda.get_device_properties(0).multi_processor_count // (b * Hkv)) + 1)   # 32 blocks per SM and more
    for n_rows in (40, 571, runs_of_blocks):
        for first in (lengths - n_rows, rng.integers(-80, 60, lengths.shape), np.full(lengths.shape, -16), np.full(lengths.shape, -n_rows), np.full(lengths.shape, 3)):
            K, V = (torch.full((b, Hkv, n_rows, d), float("nan"), dtype=cache.t, device="cuda") for _ in range(2))
            handle.paged_read(cache.desc, cache.K, cache.V, dev_i32(lengths), cache.table, n_rows, K, V, first=dev_i32(first))
            torch.cuda.synchronize()
            starts = np.broadcast_to(first.reshape(b, -1), (b, Hkv))
            for got, is_key in ((K, True), (V, False)):
                got = got.float().cpu().numpy()
                for i in range(b):
                    for h in range(Hkv):
                        want = np.zeros((n_rows, d), np.float32)
                        lo, hi = max(0, int(starts[i, h])), min(int(per[i, h]), int(starts[i, h]) + n_rows)
                        if hi > lo:
                            want[lo - starts[i, h]:hi - starts[i, h]] = host[is_key, i, h][lo:hi]
                        assert np.array_equal(got[i, h], want), (n_rows, i, h)
    assert handle.poll_status() == rk.RESTKV_OK


# ---- each attention kernel against the bits that the header states for it --------------------------------------------------------------

def attend_closely(handle, cache, lengths, Q, kernel, hidden=(), tokens=None, note=""):
    """One call against 64 bits, within what the header says is rounded in that kernel ("few" tokens, "chunk", "fp32") plus fp32 sums and the
    output's own rounding.  hidden: table slots (sequence, slot) whose page number is bad; tokens: the query tokens that are looked at."""
    b, Hq, Hkv, d, R, t = cache.batch, cache.Hq, cache.Hkv, cache.d, cache.R, Q.shape[2]
    G = Hq // Hkv
    out = torch.full((b, Hq, t, d), float("nan"), dtype=cache.t, device="cuda")
    lse = torch.full((b, Hq, t), float("nan"), device="cuda")
    ws = torch.full((handle.paged_workspace_bytes(cache.desc, t),), 255, dtype=torch.uint8, device="cuda")
    table = cache.table.clone()
    for i, slot in hidden:
        table[i, slot] = (-1, cache.n_pages, 2 ** 31 - 1)[slot % 3]
    handle.set_kernel_path(1 if kernel == "fp32" else 0)
    try:
        handle.paged_attend(cache.desc, t, Q, cache.K, cache.V, dev_i32(lengths), table, out, ws, lse=lse)
    finally:
        handle.set_kernel_path(0)
    torch.cuda.synchronize()
    assert handle.poll_status() == (rk.ERR_INVALID_ARG if hidden else rk.RESTKV_OK), note
    got_o, got_l, q64 = np64(out), np64(lse), np64(Q)
    for i in range(b):
        n = int(lengths[i])
        there = np.array([(i, r // R) not in hidden for r in range(n)], bool)
        for h in range(Hkv):
            K, k_steps = cache.rows(cache.K, True, i, h, n)
            V, v_steps = cache.rows(cache.V, False, i, h, n)
            # what K's products are made of: |K| itself, or offsets and up to 15 steps of a group
            K_parts = np.abs(K) + 30 * k_steps
            for hq in range(h * G, h * G + G):
                for j in range(t) if tokens is None else tokens:
                    see = np.flatnonzero(there[: max(0, n - (t - 1 - j))])
                    if len(see) == 0:
                        assert np.all(got_o[i, hq, j] == 0) and np.isneginf(got_l[i, hq, j]), note
                        continue
                    q, v, step = q64[i, hq, j], V[see], v_steps[see]
                    s = (K[see] @ q) * cache.scale
                    # fp32 sums of d terms in the tensor cores' order: 2^-19 of their sizes; chunks keep steps of K down to 2^-16 of the
                    # largest of 128 rows; the cap's tanh has a relative error of 2^-21, or under small caps 2^-22 of the cap
                    parts = K_parts[see].max(0) if kernel == "chunk" and cache.fmt == "int4" else K_parts[see]
                    dl = 2.0 ** -19 * (parts @ np.abs(q)).max() * cache.scale + 2.0 ** -20
                    if kernel == "chunk" and cache.fmt == "int4":
                        dl += 2.0 ** -16 * (k_steps.max(0) @ np.abs(q)) * cache.scale
                    if cache.cap:
                        dl += 2.0 ** -19 * np.abs(s).max()
                        s = cache.cap * np.tanh(s / cache.cap)
                    top = s.max()
                    w = np.exp(s - top)
                    l = top + math.log(w.sum())
                    w /= w.sum()
                    o, mass = w @ v, w @ np.abs(v)
                    if kernel == "fp32":
                        bits = 0.0
                    elif cache.fmt == "bf16":
                        bits = (2.0 ** -16 if kernel == "few" else 2.0 ** -8) * mass
                    elif kernel == "few":     # weight * step in f16 meets a code; below 2^-19 of the largest such product (2^5) an f16's last place
                        bits = 2.0 ** -11 * (w @ (15 * step)) + len(see) * 15 * 2.0 ** -30 * w.max() * step.max()
                    else:                     # weights and values in f16, both in the range of their tile
                        bits = 2.0 ** -10 * mass + 2.0 ** -13 * step.max() + len(see) * 2.0 ** -30 * w.max() * np.abs(v).max()
                    bound = bits + (2.1 * dl + 2.0 ** -18) * mass + (2.0 ** -8 if cache.dtype == "bf16" else 2.0 ** -24) * np.abs(o) + 1e-30
                    err = np.abs(got_o[i, hq, j] - o)
                    assert np.all(err <= bound), "%s: out %.3f of the bound (%s)" % (note, float((err / bound).max()), (i, hq, j))
                    assert abs(got_l[i, hq, j] - l) <= dl + 2.0 ** -20 * abs(l) + 2.0 ** -18, "%s: lse off by %.3g for %.3g" % (note, got_l[i, hq, j] - l, dl)
    return out


CLOSELY = [("few", 1), ("few", 3), ("chunk", 200), ("fp32", 1), ("fp32", 70)]     # kernel, tokens (of 8 query heads over 2 KV heads)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group", [("bf16", 0), ("int4", 32), ("int4", 64), ("int4", 128)])
@pytest.mark.parametrize("kernel,t", CLOSELY)
@pytest.mark.parametrize("cap", [0.0, 3.0, 50.0, 1e3, 1e5, 1e6, 1e8, 1e20, 3e38])
def test_attend_under_caps_of_any_size(handle, fmt, group, kernel, t, cap):
    """A cap far above the logits leaves them as they are, one near them bends them: in every kernel, logits with and without others near the cap
    beside them."""
    rng = np.random.default_rng(22)
    cache = Cache(rng, 1, 8, 2, 128, fmt, 16, 22, group, softcap=cap)
    cache.fill(handle, rng, [340])
    for scale in (0.1, 2.0) + ((cap,) if 1e3 <= cap <= 1e6 else ()):
        q = rng.standard_normal((1, 8, t, 128))
        q[:, :1 if scale == cap else 8] *= scale        # or one head's logits reach the cap, in the same tiles as those of the others
        attend_closely(handle, cache, [340], to_dev(q, cache.t), kernel, tokens=[0, t // 2, t - 1], note="%s, q %g" % (kernel, scale))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group", [("bf16", 0), ("int4", 32), ("int4", 128)])
@pytest.mark.parametrize("kernel,t", CLOSELY)
@pytest.mark.parametrize("page_rows", [16, 48])
@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_rows_of_bad_pages_are_not_seen(handle, fmt, group, kernel, t, page_rows, cap):
    """Rows whose page number is outside the pool carry no weight, in every kernel alike; queries that see no others get 0 and -inf."""
    rng = np.random.default_rng(23)
    cache = Cache(rng, 2, 8, 2, 128, fmt, page_rows, -(-340 // page_rows), group, softcap=cap)
    lengths = [340, 210]
    cache.fill(handle, rng, lengths)
    hidden = {(0, 1), (0, 2), (0, 6), (0, 339 // page_rows), (1, 0), (1, 3), (1, 4)} | ({(1, s) for s in range(5)} if page_rows == 16 else set())
    tokens = sorted({0, 5, t // 3, t // 2, t - 1} & set(range(t)))
    attend_closely(handle, cache, lengths, to_dev(rng.standard_normal((2, 8, t, 128)), cache.t), kernel, hidden, tokens)
    only = [min(lengths[0], 3 * page_rows), lengths[1]]      # a sequence that ends with its bad pages
    attend_closely(handle, cache, only, to_dev(rng.standard_normal((2, 8, t, 128)), cache.t), kernel, {(0, 0), (0, 1), (0, 2), (1, 4)}, tokens)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_rows_of_bad_pages_among_many_sequences(handle, fmt):
    """Chunks of more tiles than the device has SMs: units that one block takes whole, several in a row, and units that blocks share."""
    rng = np.random.default_rng(24)
    b = 40
    cache = Cache(rng, b, 4, 2, 64, fmt, 16, 30, 32 if fmt == "int4" else 0)
    lengths = [131 + (97 * i) % 340 for i in range(b)]
    cache.fill(handle, rng, lengths)
    hidden = {(i, int(s)) for i in range(1, b, 3) for s in rng.integers(0, lengths[i] // 16, 2)}
    attend_closely(handle, cache, lengths, to_dev(rng.standard_normal((b, 4, 131, 64)), cache.t), "chunk", hidden, [0, 17, 100, 130])


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group", [("bf16", 0), ("int4", 64)])
@pytest.mark.parametrize("b,Hq,Hkv,t,n", [(1, 8, 2, 1, 3000), (1, 32, 8, 1, 40000), (1, 8, 2, 200, 3000), (4, 8, 2, 300, 600)])
def test_paged_waits_that_run_out(handle, fmt, group, b, Hq, Hkv, t, n):
    """A wait limit of one SM clock in the tensor-core kernels of few tokens (in clusters, dealt out) and of many: whichever waits run out, the
    call returns by itself, with the timeout status or with its results, and the next one has them."""
    rng = np.random.default_rng(25)
    cache = Cache(rng, b, Hq, Hkv, 128, fmt, 64, -(-n // 64), group)
    lengths = [n - 100 * i for i in range(b)]
    cache.fill(handle, rng, lengths)
    Q = to_dev(rng.standard_normal((b, Hq, t, 128)), torch.bfloat16)
    ws = torch.empty(handle.paged_workspace_bytes(cache.desc, t), dtype=torch.uint8, device="cuda")

    def call():
        out, lse = torch.empty_like(Q), torch.empty(b, Hq, t, device="cuda")
        handle.paged_attend(cache.desc, t, Q, cache.K, cache.V, dev_i32(lengths), cache.table, out, ws, lse=lse)
        torch.cuda.synchronize()
        return handle.poll_status(), out, lse

    status, want, want_lse = call()
    assert status == rk.RESTKV_OK
    for _ in range(5):
        try:
            handle.set_wait_limit(1)
            status, out, lse = call()
        finally:
            handle.set_wait_limit(2_000_000_000)
        assert status in (rk.RESTKV_OK, rk.ERR_TIMEOUT)
        if status == rk.RESTKV_OK:
            assert torch.equal(out, want) and torch.equal(lse, want_lse)
        status, out, lse = call()
        assert status == rk.RESTKV_OK and torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("dtype,fmt", [(rk.BF16, rk.PAGES_BF16), (rk.BF16, rk.PAGES_INT4), (rk.F32, rk.PAGES_F32), (rk.F32, rk.PAGES_INT4)])
@pytest.mark.parametrize("b,Hq,Hkv,d", [(1, 32, 8, 128), (1, 8, 8, 64), (3, 6, 2, 96), (8, 16, 1, 256), (1, 1, 1, 32), (70, 4, 4, 128)])
@pytest.mark.parametrize("width", [1, 3, 2000])
def test_workspaces_serve_calls_of_fewer_tokens(dtype, fmt, b, Hq, Hkv, d, width):
    """Sizes never fall as the tokens grow, and never pass what the blocks of one device can leave: two parts of 256 query rows per SM."""
    lib = rk.load_library()
    cache = rk.make_paged(b, Hq, Hkv, d, fmt, 64, b * width, width, 32 if fmt == rk.PAGES_INT4 else 0, dtype)
    before = 0
    for t in list(range(1, 200)) + [2 ** k + x for k in range(8, 17) for x in (-1, 0, 1) if (2 ** k + x) * Hq // Hkv < 200000]:
        size = lib.restkv_paged_workspace_bytes(ctypes.byref(cache), t)
        assert size % 256 == 0 and before <= size <= 148 * (2 * 256 * (d + 2) * 4 + 16) + 256, t
        before = size


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "f32", "int4-bf16"])
def test_one_workspace_for_all_calls_of_a_size_and_fewer(handle, fmt):
    rng = np.random.default_rng(26)
    dtype = "f32" if fmt.endswith("f32") else "bf16"
    cache = Cache(rng, 1, 8, 8, 64, fmt.split("-")[0], 16, 30, 32 if fmt.startswith("int4") else 0, dtype)
    cache.fill(handle, rng, [470])
    size = handle.paged_workspace_bytes(cache.desc, 50)
    memory = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    for t in (50, 49, 17, 6, 5, 4, 3, 1):
        Q = to_dev(rng.standard_normal((1, 8, t, 64)), cache.t)
        out, want = torch.empty_like(Q), torch.empty_like(Q)
        handle.paged_attend(cache.desc, t, Q, cache.K, cache.V, dev_i32([470]), cache.table, out, memory[:size])
        own = torch.empty(handle.paged_workspace_bytes(cache.desc, t), dtype=torch.uint8, device="cuda")
        handle.paged_attend(cache.desc, t, Q, cache.K, cache.V, dev_i32([470]), cache.table, want, own)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    assert handle.poll_status() == rk.RESTKV_OK
    assert bool((memory[size:] == 0xA5).all())


@pytest.mark.gpu
@pytest.mark.parametrize("path", [rk.PATH_TENSOR_CORE, 3])
@pytest.mark.parametrize("fmt,d,t,on_tensor_cores", [("f32", 128, 1, False), ("int4-f32", 64, 70, False), ("bf16", 96, 1, False), ("int4-bf16", 32, 200, False), ("bf16", 128, 1, True),
                                                     ("int4-bf16", 64, 1, True), ("bf16", 256, 40, True), ("int4-bf16", 128, 400, True)])
def test_attend_where_the_tensor_cores_are_required(handle, path, fmt, d, t, on_tensor_cores):
    rng = np.random.default_rng(27)
    cache = Cache(rng, 1, 8, 2, d, fmt.split("-")[0], 16, 32, 32 if fmt.startswith("int4") else 0, "f32" if fmt.endswith("f32") else "bf16")
    cache.fill(handle, rng, [500])
    Q = to_dev(rng.standard_normal((1, 8, t, d)), cache.t)
    out, want = torch.full_like(Q, 7.0), torch.empty_like(Q)
    ws = torch.empty(handle.paged_workspace_bytes(cache.desc, t), dtype=torch.uint8, device="cuda")
    handle.paged_attend(cache.desc, t, Q, cache.K, cache.V, dev_i32([500]), cache.table, want, ws)
    launches = handle.launch_count()
    handle.set_kernel_path(path)
    try:
        if on_tensor_cores:
            handle.paged_attend(cache.desc, t, Q, cache.K, cache.V, dev_i32([500]), cache.table, out, ws)
        else:
            with pytest.raises(rk.RestKVError) as e:
                handle.paged_attend(cache.desc, t, Q, cache.K, cache.V, dev_i32([500]), cache.table, out, ws)
            assert e.value.status == rk.ERR_UNSUPPORTED and handle.launch_count() == launches
    finally:
        handle.set_kernel_path(0)
    torch.cuda.synchronize()
    assert torch.equal(out, want) if on_tensor_cores else bool((out == 7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group,kernel", [("bf16", 0, "chunk"), ("int4", 64, "chunk"), ("bf16", 0, "fp32"), ("int4", 32, "fp32")])
def test_more_query_rows_than_a_grid_has_in_its_second_dimension(handle, fmt, group, kernel):
    """4100 tokens of 64 query heads over one KV head: 262 400 query rows, appended with their queries and attended over."""
    rng = np.random.default_rng(28)
    t, n = 4100, 4160
    cache = Cache(rng, 1, 64, 1, 64, fmt, 64, 65, group)
    cache.fill(handle, rng, [n])
    Q = torch.randn(1, 64, t, 64, generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(cache.t)
    K, V, k, v = (torch.empty(1, 1, t, 64, dtype=cache.t, device="cuda") for _ in range(4))
    handle.paged_read(cache.desc, cache.K, cache.V, dev_i32([n]), cache.table, t, K, V, first=dev_i32([n - t]))
    other = cache.K.clone(), cache.V.clone()
    Q_out = torch.empty_like(Q)
    handle.paged_append(cache.desc, t, K, V, *other, dev_i32([n]), cache.table, Q=Q, Q_out=Q_out)
    handle.paged_read(cache.desc, *other, dev_i32([n]), cache.table, t, k, v, first=dev_i32([n - t]))
    assert torch.equal(Q_out, Q)
    if fmt == "bf16":
        assert torch.equal(k, K) and torch.equal(v, V)
    attend_closely(handle, cache, [n], Q, kernel, tokens=[0, 1777, 4095, 4099])


# ---- a length per head ------------------------------------------------------------------------------------------------------------------

def by_head(cache):
    """The same pool as pages of one head, batch * n_kv_heads sequences: its description and the table for it, as the header says."""
    d = cache.desc
    one = rk.make_paged(d.batch * d.n_kv_heads, d.n_q_heads // d.n_kv_heads, 1, d.head_dim, d.page_format, d.page_rows, d.n_pages * d.n_kv_heads, d.table_width,
                        d.group, d.dtype)
    table = cache.table[:, None, :] * d.n_kv_heads + torch.arange(d.n_kv_heads, dtype=torch.int32, device="cuda")[None, :, None]
    return one, table.reshape(-1, d.table_width).contiguous()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group", [("bf16", 0), ("int4", 64)])
def test_rows_kept_under_budgets_of_heads_go_into_pages(handle, fmt, group):
    """restkv_evict_budgets leaves a head's kept rows first: they go in head by head, and after that every call takes lengths per head."""
    b, Hq, Hkv, d, n_kv, w, S = 2, 8, 4, 128, 400, 32, 90
    rng = np.random.default_rng(29)
    K, V = (to_dev(rng.standard_normal((b, Hkv, n_kv, d)), torch.bfloat16) for _ in range(2))
    Q = to_dev(rng.standard_normal((b, Hq, w, d)), torch.bfloat16)
    budgets = np.array([[90, 1, 64, 33], [17, 200, 48, 5]])
    lengths = np.minimum(budgets, S)
    shape = rk.make_shape(b, Hq, Hkv, d, n_kv, w)
    ws = torch.empty(handle.workspace_bytes(shape, S), dtype=torch.uint8, device="cuda")
    indices = torch.empty(b, Hkv, S, dtype=torch.int32, device="cuda")
    K_out, V_out = (torch.full((b, Hkv, S, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    handle.evict_budgets(shape, Q, K, V, 0.9, rk.fixed_pool(5), dev_i32(budgets), S, indices, K_out, V_out, ws)

    cache = Cache(rng, b, Hq, Hkv, d, fmt, 16, 8, group, per_head=True)
    one, table = by_head(cache)
    n = dev_i32(lengths)
    handle.paged_append(one, S, K_out.view(b * Hkv, 1, S, d), V_out.view(b * Hkv, 1, S, d), cache.K, cache.V, n.view(-1), table, counts=n.view(-1))
    assert handle.poll_status() == rk.RESTKV_OK
    idx = indices.cpu().numpy()
    for i in range(b):
        for h in range(Hkv):
            rows = np64(K[i, h])[idx[i, h, :lengths[i, h]]]
            got, steps = cache.rows(cache.K, True, i, h, int(lengths[i, h]))
            assert np.all(np.abs(got - rows) <= 0.5 * steps + (2.0 ** -20 * np.abs(rows).max() if group else 0.0))
    check_attention(handle, rng, cache, lengths, None, 1)
    # generated tokens: one row more in every head
    new = [to_dev(rng.standard_normal((b, Hkv, 3, d)), torch.bfloat16) for _ in range(2)]
    handle.paged_append(cache.desc, 3, *new, cache.K, cache.V, n + 3, cache.table)
    k, v = (torch.empty(b, Hkv, 3, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    handle.paged_read(cache.desc, cache.K, cache.V, n + 3, cache.table, 3, k, v, first=n)
    torch.cuda.synchronize()
    for got, want in zip((k, v), new):
        span = want.float().unflatten(-1, (-1, group or d))
        step = (span.amax(-1) - span.amin(-1))[..., None].expand(span.shape).flatten(-2) * ((1 + 2.0 ** -6) / 15 if group else 0.0)
        assert bool(((got.float() - want.float()).abs() <= 0.5 * step + (2.0 ** -8 * want.float().abs() + 2.0 ** -8 * 0.2 if group else 0.0)).all())
    check_attention(handle, rng, cache, lengths + 3, None, 3)
    assert handle.poll_status() == rk.RESTKV_OK


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "f32", "int4-bf16", "int4-f32"])
@pytest.mark.parametrize("t", [1, 5, 70])
def test_append_with_lengths_per_head(handle, fmt, t):
    """Byte for byte what the same rows give head by head, rotated, with counts, and rows of a bad page or past the table left out."""
    b, Hq, Hkv, d, R = 3, 6, 3, 64, 16
    rng = np.random.default_rng(30)
    dtype = "f32" if fmt.endswith("f32") else "bf16"
    fmt = fmt.split("-")[0]
    cache = Cache(rng, b, Hq, Hkv, d, fmt, R, 10, 32 if fmt == "int4" else 0, dtype, per_head=True)
    one, table = by_head(cache)
    counts = np.array([t, max(0, t - 4), t // 2])
    lengths = np.array([[70, 160, 101], [87, 80, 159], [150, 71, 90]])
    K, V = (to_dev(rng.standard_normal((b, Hkv, t, d)), cache.t) for _ in range(2))
    Q = to_dev(rng.standard_normal((b, Hq, t, d)), cache.t)
    positions = rng.integers(0, 300, (b, t)).astype(np.int32)
    cos, sin = tables(300, d)
    rotation = rk.make_rotation(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), d)
    want_K, want_V, q = cache.K.clone(), cache.V.clone(), torch.empty_like(Q)
    handle.paged_append(cache.desc, t, K, V, cache.K, cache.V, dev_i32(lengths), cache.table, counts=dev_i32(counts), positions=dev_i32(positions), rotation=rotation, Q=Q, Q_out=q)
    handle.paged_append(one, t, K.view(b * Hkv, 1, t, d), V.view(b * Hkv, 1, t, d), want_K, want_V, dev_i32(lengths.reshape(-1)), table,
                        counts=dev_i32(np.repeat(counts, Hkv)), positions=dev_i32(np.repeat(positions, Hkv, 0)), rotation=rotation)
    torch.cuda.synchronize()
    assert handle.poll_status() == rk.RESTKV_OK
    assert torch.equal(cache.K, want_K) and torch.equal(cache.V, want_V)
    assert bool((cache.K != 255).any())
    for i in range(b):
        turned = rotate(np64(Q[i]), positions[i], cos, sin, d, False)
        assert np.all(np.abs(np64(q[i]) - turned)[:, :counts[i]] <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(turned[:, :counts[i]]) + 2.0 ** -20 * np.abs(turned).max())
        assert bool((q[i, :, counts[i]:] == 0).all())
    # rows without a place: of the heads that have none, nothing; the others' as before
    lengths[0, 1], lengths[2, 0] = 161, 2
    cache.table[1, 4] = cache.n_pages
    one, table = by_head(cache)
    handle.paged_append(cache.desc, t, V, K, cache.K, cache.V, dev_i32(lengths), cache.table, counts=dev_i32(counts))
    assert handle.poll_status() == rk.ERR_INVALID_ARG
    handle.paged_append(one, t, V.view(b * Hkv, 1, t, d), K.view(b * Hkv, 1, t, d), want_K, want_V, dev_i32(lengths.reshape(-1)), table, counts=dev_i32(np.repeat(counts, Hkv)))
    assert handle.poll_status() == rk.ERR_INVALID_ARG
    assert torch.equal(cache.K, want_K) and torch.equal(cache.V, want_V)


# ---- values, long caches and unlike groups, within the stated bits ------------------------------------------------------------------------

# kernel, batch, query heads, KV heads, head_dim, page rows, lengths, tokens, the tokens looked at
CLOSE = [("few", 1, 8, 2, 128, 64, [17000], 1, [0]), ("few", 3, 8, 2, 128, 16, [300, 1, 6001], 1, [0]), ("few", 1, 16, 1, 128, 32, [5300], 1, [0]), ("few", 2, 4, 1, 64, 16, [900, 33], 4, [0, 3]),
         ("few", 1, 4, 2, 256, 48, [2500], 1, [0]), ("few", 1, 8, 2, 256, 16, [1100], 6, [0, 5]), ("few", 1, 12, 4, 128, 16, [700], 9, [0, 4, 8]),
         ("chunk", 1, 8, 2, 128, 64, [6000], 200, [0, 99, 199]), ("chunk", 2, 4, 4, 64, 16, [900, 333], 333, [0, 150, 332]), ("chunk", 1, 16, 1, 128, 16, [2100], 2100, [0, 255, 1024, 2099]),
         ("fp32", 1, 8, 2, 128, 64, [6000], 1, [0]), ("fp32", 2, 6, 2, 96, 16, [700, 65], 9, [0, 8])]


@pytest.mark.gpu
@pytest.mark.parametrize("spec", CLOSE)
@pytest.mark.parametrize("fmt,group", [("bf16", 0), ("int4", 32), ("int4", 64), ("int4", 128)])
@pytest.mark.parametrize("q_scale", [0.3, 2.0])
def test_attend_within_the_stated_bits(handle, spec, fmt, group, q_scale):
    kernel, b, Hq, Hkv, d, R, lengths, t, tokens = spec
    if group and d % group:
        pytest.skip("no such group in this head_dim")
    rng = np.random.default_rng(31)
    cache = Cache(rng, b, Hq, Hkv, d, fmt, R, -(-max(lengths) // R), group)
    cache.fill(handle, rng, lengths)
    attend_closely(handle, cache, lengths, to_dev(rng.standard_normal((b, Hq, t, d)) * q_scale, cache.t), kernel, tokens=tokens)


@pytest.mark.gpu
@pytest.mark.parametrize("group", [32, 64])
@pytest.mark.parametrize("kernel,t", CLOSELY)
@pytest.mark.parametrize("ratio", [2.0 ** -8, 2.0 ** -16, 2.0 ** -24])
def test_attend_over_groups_of_unlike_steps(handle, group, kernel, t, ratio):
    """Groups of V whose values are far smaller than the first one's keep the bits that the header promises them."""
    rng = np.random.default_rng(32)
    cache = Cache(rng, 1, 8, 2, 128, "int4", 16, 40, group)
    K, V = rng.standard_normal((2, 1, 2, 600, 128))
    V *= ratio ** (np.arange(128) // group)
    handle.paged_append(cache.desc, 600, to_dev(K, cache.t), to_dev(V, cache.t), cache.K, cache.V, dev_i32([600]), cache.table)
    attend_closely(handle, cache, [600], to_dev(rng.standard_normal((1, 8, t, 128)), cache.t), kernel, tokens=[0, t - 1])


@pytest.mark.gpu
@pytest.mark.parametrize("group", [32, 64, 128])
def test_attend_keeps_its_bits_over_long_caches(handle, group):
    """One token over 524 288 rows of 4 bits: what is rounded are the weights and the output, each on its own, so that the error of all outputs
    together is no more than independent roundings give; nothing adds up along the rows."""
    Hkv, G, d, n, R = 8, 2, 128, 524288, 256
    g = torch.Generator("cuda").manual_seed(33)
    cache = rk.make_paged(1, Hkv * G, Hkv, d, rk.PAGES_INT4, R, n // R, n // R, group)
    pages = [torch.empty(n // R * handle.paged_page_bytes(cache), dtype=torch.uint8, device="cuda") for _ in range(2)]
    table, lengths = torch.randperm(n // R, generator=g, device="cuda").to(torch.int32), dev_i32([n])
    handle.paged_append(cache, n, *(torch.randn(1, Hkv, n, d, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2)), *pages, lengths, table)
    Q = torch.randn(1, Hkv * G, 1, d, generator=g, device="cuda").to(torch.bfloat16)
    out = torch.empty_like(Q)
    ws = torch.empty(handle.paged_workspace_bytes(cache, 1), dtype=torch.uint8, device="cuda")
    handle.paged_attend(cache, 1, Q, *pages, lengths, table, out, ws)
    # the rows as single precision has them: offset + step * code has few bits
    exact = rk.make_paged(1, Hkv * G, Hkv, d, rk.PAGES_INT4, R, n // R, n // R, group, rk.F32)
    K, V = (torch.empty(1, Hkv, n, d, device="cuda") for _ in range(2))
    handle.paged_read(exact, *pages, lengths, table, n, K, V)
    assert handle.poll_status() == rk.RESTKV_OK
    err, size, rounded = 0.0, 0.0, 0.0
    for h in range(Hkv):
        w = torch.softmax(Q[0, h * G:h * G + G, 0].double() @ K[0, h].double().T / math.sqrt(d), -1)
        v = V[0, h].double()
        o = w @ v
        spread = v.unflatten(-1, (-1, group))
        span = (spread.amax(-1) - spread.amin(-1)).repeat_interleave(group, -1)          # at most 15 steps, by which a weight is rounded
        err += float(((out[0, h * G:h * G + G, 0].double() - o) ** 2).sum())
        size += float((o ** 2).sum())
        rounded += float(((w ** 2) @ (span * (15.0 / 14.0)) ** 2).sum())               # (a span of 14 steps of 15 is the least that codes have)
    # half a place of the output's 8 bits and of the weights' 11, evenly spread: 2^-7 / sqrt(12) and 2^-10 / sqrt(12)
    bound = 2.0 ** -14 / 12 * size + 2.0 ** -20 / 12 * rounded
    assert err <= 1.2 * bound, (err / size) ** 0.5
