"""Cross attention: decoder tokens over an encoder's rows, shared by the hypotheses of a source, against a plain implementation in 64 bits."""
import ctypes
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2605_08840_b200 import binding as rk
from paper_2605_08840_b200 import build as rk_build

NEG_INF = float("-inf")


@pytest.fixture(scope="module")
def handle():
    h = rk.Handle()
    yield h
    h.close()


def dev_i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def make(sources, beams, Hq, Hkv, d, t, m, dtype, seed, q_scale=1.0, layout="rows"):
    """Q, K, V on the device.  layout: "rows" as one projection leaves them ([.., n, heads, d]), "dense" contiguous, "wide" with gaps between rows."""
    g = torch.Generator("cuda").manual_seed(seed)
    b = sources * beams
    Q = torch.randn(b, t, Hq, d, generator=g, device="cuda") * q_scale
    kv = torch.randn(sources, m, 2 * Hkv, d, generator=g, device="cuda")
    if layout == "rows":
        Q, kv = Q.to(dtype).transpose(1, 2), kv.to(dtype).transpose(1, 2)
    elif layout == "dense":
        Q, kv = Q.transpose(1, 2).to(dtype).contiguous(), kv.transpose(1, 2).to(dtype).contiguous()
    else:
        wide = torch.full((sources, 2 * Hkv, m, d + 24), float("nan"), dtype=dtype, device="cuda")
        wide[..., :d] = kv.transpose(1, 2)
        Q, kv = Q.transpose(1, 2).to(dtype).contiguous(), wide[..., :d]
    return Q, kv[:, :Hkv], kv[:, Hkv:]


def plain(Q, K, V, lengths, counts, scale):
    """out, lse, sum of weights times |v|, size of the logits, in 64 bits; lengths [sources, KV heads], counts [sequences]."""
    b, Hq, t, d = Q.shape
    S, Hkv, m, _ = K.shape
    beams, G = b // S, Hq // Hkv
    out, mass = (torch.zeros(b, Hq, t, d, dtype=torch.float64, device="cuda") for _ in range(2))
    lse, size = torch.full((b, Hq, t), NEG_INF, dtype=torch.float64, device="cuda"), torch.zeros(b, Hq, t, dtype=torch.float64, device="cuda")
    for i in range(b):
        c = int(counts[i])
        for h in range(Hkv):
            n = int(lengths[i // beams, h])
            if n == 0 or c == 0:
                continue
            k, v = K[i // beams, h, :n].double(), V[i // beams, h, :n].double()
            q = Q[i, h * G:(h + 1) * G, :c].double()
            s = q @ k.T * scale
            w = torch.softmax(s, -1)
            at = (i, slice(h * G, (h + 1) * G), slice(0, c))
            lse[at], out[at], mass[at] = torch.logsumexp(s, -1), w @ v, w @ v.abs()
            size[at] = (q.abs() @ k.abs().T).amax(-1) * scale
    return out, lse, mass, size


def check(handle, Q, K, V, lengths=None, counts=None, scale=0.0, note="", closely=False):
    b, Hq, t, d = Q.shape
    S, Hkv, m, _ = K.shape
    lengths_np = np.full((S, Hkv), m) if lengths is None else np.broadcast_to(np.asarray(lengths).reshape(S, -1), (S, Hkv))
    per_head = lengths is not None and np.asarray(lengths).ndim == 2
    desc = rk.make_cross(S, b // S, Hq, Hkv, d, m, rk.F32 if Q.dtype == torch.float32 else rk.BF16, per_head, scale)
    out, lse = torch.full((b, Hq, t, d), float("nan"), dtype=Q.dtype, device="cuda"), torch.full((b, Hq, t), float("nan"), device="cuda")
    ws = torch.full((handle.cross_workspace_bytes(desc, t),), 255, dtype=torch.uint8, device="cuda")
    handle.cross_attend(desc, t, Q, K, V, out, ws, lengths=None if lengths is None else dev_i32(lengths), lse=lse, counts=None if counts is None else dev_i32(counts))
    torch.cuda.synchronize()
    assert handle.poll_status() == rk.RESTKV_OK
    o, l, mass, size = plain(Q, K, V, np.clip(lengths_np, 0, m), np.full(b, t) if counts is None else np.clip(counts, 0, t), scale or 1 / math.sqrt(d))
    empty = torch.isneginf(l)
    assert torch.equal(torch.isneginf(lse), empty), note
    assert bool((out[empty] == 0).all()), note
    # a logit is an fp32 sum of d products: at most 2^-19 of the sum of their sizes, and so is the weights' exponent twice
    dl = 2.0 ** -19 * size + 2.0 ** -20
    if Q.dtype == torch.float32:
        bound = 2.0 ** -17 * mass + 4 * dl[..., None] * mass + 1e-30
    else:
        # weights of one bf16 (closely: of two, 2^-17) or fp32, and an output rounded once
        bound = ((2.0 ** -16 if closely else 2.0 ** -8) + 2.0 ** -15) * mass + 4 * dl[..., None] * mass + 2.0 ** -8 * o.abs() + 1e-30
    err = (out.double() - o).abs()
    assert bool((err <= bound).all()), "%s: out %.3f of the bound" % (note, float((err / bound).max()))
    ok = ~empty
    assert bool(((lse.double() - l).abs()[ok] <= (2 * dl + 2.0 ** -21 * l.abs() + 2.0 ** -18)[ok]).all()), note
    return out, lse


# sources, beams, query heads, KV heads, head_dim, tokens, lengths (the longest is n_rows), counts
CROSS = [(1, 1, 1, 1, 128, 1, [1], None), (1, 4, 8, 2, 128, 1, [15], None), (2, 1, 4, 4, 64, 1, [16, 17], None), (3, 5, 8, 8, 64, 1, [260, 0, 33], None),
         (1, 4, 32, 8, 128, 1, [1500], None), (2, 3, 6, 2, 128, 3, [100, 129], [3, 1, 2, 0, 3, 3]), (1, 1, 16, 1, 128, 2, [700], None), (2, 8, 8, 2, 64, 1, [3000, 77], None),
         (1, 2, 4, 1, 96, 5, [200], None), (2, 2, 4, 2, 256, 2, [77, 300], None), (1, 3, 2, 2, 40, 1, [64], None), (1, 1, 2, 2, 8, 70, [90], None),
         (1, 1, 4, 1, 128, 70, [300], None), (2, 1, 8, 2, 64, 200, [500, 129], [200, 13]), (1, 1, 32, 8, 128, 300, [1000], None), (3, 2, 4, 2, 128, 129, [128, 0, 257], None),
         (1, 20, 12, 4, 128, 1, [999], None), (40, 1, 8, 8, 64, 1, list(range(1, 41)), None), (1, 1, 2, 1, 128, 1000, [1], None), (2, 64, 4, 2, 64, 2, [100, 600], None)]


@pytest.mark.gpu
@pytest.mark.parametrize("spec", CROSS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["rows", "dense", "wide"])
def test_cross(handle, spec, dtype, layout):
    S, beams, Hq, Hkv, d, t, lengths, counts = spec
    m = max(lengths) + (3 if layout == "wide" else 0)
    Q, K, V = make(S, beams, Hq, Hkv, d, t, m, dtype, Hq + d + t, 1.5, layout)
    for b, n in enumerate(lengths):              # what lies behind a source's rows is nobody's business
        K[b, :, n:], V[b, :, n:] = float("nan"), float("nan")
    if counts:
        for i, n in enumerate(counts):
            Q[i, :, n:] = float("nan")
    check(handle, Q, K, V, None if min(lengths) == m else lengths, counts)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("t", [1, 150])
def test_cross_lengths_per_head(handle, dtype, t):
    Q, K, V = make(2, 2, 8, 4, 128, t, 310, dtype, 5)
    lengths = [[310, 0, 17, 129], [1, 128, 300, -4]]
    for b in range(2):
        for h in range(4):
            K[b, h, max(0, lengths[b][h]):], V[b, h, max(0, lengths[b][h]):] = float("nan"), float("inf")
    check(handle, Q, K, V, lengths)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("t", [1, 4, 150])
@pytest.mark.parametrize("q_scale", [0.0, 40.0, 1000.0])
def test_cross_extreme_logits(handle, dtype, t, q_scale):
    Q, K, V = make(2, 2, 8, 2, 128, t, 700, dtype, 6, q_scale)
    check(handle, Q, K, V, [700, 333])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("t", [1, 3, 400])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fall", [False, True])
def test_cross_logits_that_grow(handle, dtype, t, d, fall):
    """Rows whose logits grow from one to the next by far more than a rescaling leaves room for, and the other way round."""
    Q, K, V = make(1, 2, 4, 2, d, t, 900, dtype, 7, 1.0, "dense")
    ramp = torch.linspace(0.0, 30.0, 900, device="cuda")
    Q[..., 0], K[..., 0] = 8.0, (ramp.flip(0) if fall else ramp).to(dtype)
    check(handle, Q, K, V)


@pytest.mark.gpu
@pytest.mark.parametrize("t", [1, 200])
@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -20, 2.0 ** 20, 2.0 ** 100])
def test_cross_values_of_any_size(handle, t, size):
    Q, K, V = make(1, 2, 8, 2, 128, t, 500, torch.bfloat16, 8, 1.0, "dense")
    check(handle, Q, K, V * size)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("t", [1, 150])
def test_cross_one_row_for_all(handle, dtype, t):
    """Queries, keys and values expanded over sequences, heads or rows (strides of 0)."""
    Q, K, V = make(1, 1, 4, 2, 128, t, 60, dtype, 9, 1.0, "dense")
    Q3 = Q.expand(6, 4, t, 128)
    check(handle, Q3, K.expand(3, 2, 60, 128), V.expand(3, 2, 60, 128), [60, 31, 0])
    check(handle, Q[:, :1].expand(1, 4, t, 128), K[:, :1].expand(1, 2, 60, 128), V)
    check(handle, Q, K[:, :, :1].expand(1, 2, 60, 128), V[:, :, :1].expand(1, 2, 60, 128))


# one token in clusters, dealt out, of several heads; many rows alone, by few CTAs, by many; fp32 with splits and without
NOT_FINITE = [(1, 4, 8, 2, 128, 1, 1500), (1, 4, 32, 8, 128, 1, 40000), (12, 5, 16, 16, 64, 1, 2000), (2, 1, 4, 2, 128, 300, 200), (1, 1, 8, 2, 64, 300, 9000), (1, 2, 2, 1, 128, 40, 30000),
              (3, 2, 4, 2, 96, 2, 700), (80, 2, 4, 4, 40, 2, 90)]


@pytest.mark.gpu
@pytest.mark.parametrize("spec", NOT_FINITE)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("what", ["key", "keys", "query", "large", "value", "infinite"])
def test_cross_of_what_is_not_finite(handle, spec, dtype, what):
    """A NaN among the logits that count, or one of +inf, is seen in the token's outputs and log-sum-exp, and nowhere else: no token of other sources,
    heads or sequences has it, and what lies behind a length or a count has no part in it."""
    S, beams, Hq, Hkv, d, t, m = spec
    Q, K, V = make(S, beams, Hq, Hkv, d, t, m, dtype, 18, 1.0, "dense")
    G, n = Hq // Hkv, m - 17
    K[:, :, n:], V[:, :, n:] = float("nan"), float("nan")
    bad = torch.zeros(S * beams, Hq, t, dtype=torch.bool, device="cuda")      # whose logits are not numbers
    if what == "key":
        K[0, 0, n // 2, 3] = float("nan")
        bad[:beams, :G] = True
    elif what == "keys":                        # every one of them
        K[0, -1, :n] = float("nan")
        bad[:beams, -G:] = True
    elif what == "query":
        Q[-1, 1, t // 2, 5] = float("nan")
        bad[-1, 1, t // 2] = True
    elif what == "large":                       # logits of +inf for tokens that are above 0 there, of -inf for the others
        K[0, 0, n - 1, 0] = float("inf")
        bad[:beams, :G] = Q[:beams, :G, :, 0] > 0
    else:
        V[0, 0, n // 3, 2] = float("nan" if what == "value" else "inf")
    desc = rk.make_cross(S, beams, Hq, Hkv, d, m, rk.F32 if dtype == torch.float32 else rk.BF16)
    ws = torch.full((handle.cross_workspace_bytes(desc, t),), 255, dtype=torch.uint8, device="cuda")
    out, lse = torch.full((S * beams, Hq, t, d), 7.0, dtype=dtype, device="cuda"), torch.full((S * beams, Hq, t), 7.0, device="cuda")
    handle.cross_attend(desc, t, Q, K, V, out, ws, lengths=dev_i32([n] * S), lse=lse)
    torch.cuda.synchronize()
    assert handle.poll_status() == rk.RESTKV_OK
    assert torch.equal(lse.isnan(), bad)
    want = bad[..., None].expand_as(out).clone()
    if what in ("value", "infinite"):
        want[:beams, :G, :, 2] = True
    assert torch.equal(~out.isfinite() if what == "infinite" else out.isnan(), want)
    assert bool(out[~want].isfinite().all()) and bool(lse[~bad].isfinite().all())


@pytest.mark.gpu
@pytest.mark.parametrize("spec", NOT_FINITE)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_cross_of_logits_that_are_all_infinite(handle, spec, dtype):
    """Keys of -inf in one channel: tokens that are above 0 there have weights of nothing and get 0 and -inf, the others are no numbers."""
    S, beams, Hq, Hkv, d, t, m = spec
    Q, K, V = make(S, beams, Hq, Hkv, d, t, m, dtype, 19, 1.0, "dense")
    K[..., 1] = NEG_INF
    desc = rk.make_cross(S, beams, Hq, Hkv, d, m, rk.F32 if dtype == torch.float32 else rk.BF16)
    ws = torch.full((handle.cross_workspace_bytes(desc, t),), 255, dtype=torch.uint8, device="cuda")
    out, lse = torch.full((S * beams, Hq, t, d), 7.0, dtype=dtype, device="cuda"), torch.full((S * beams, Hq, t), 7.0, device="cuda")
    handle.cross_attend(desc, t, Q, K, V, out, ws, lse=lse)
    torch.cuda.synchronize()
    assert handle.poll_status() == rk.RESTKV_OK
    empty = Q[..., 1] > 0
    assert torch.equal(lse.isneginf(), empty) and torch.equal(lse.isnan(), ~empty)
    assert bool((out[empty] == 0).all()) and bool(out[~empty].isnan().all())


@pytest.mark.gpu
@pytest.mark.parametrize("spec", [(1, 4, 32, 8, 128, 1, 20000), (8, 5, 16, 16, 64, 1, 3000), (1, 1, 32, 8, 128, 600, 5000), (4, 2, 8, 2, 64, 40, 500), (2, 3, 8, 2, 64, 4, 1024)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_cross_same_bits_in_a_graph_and_on_another_stream(handle, spec, dtype):
    S, beams, Hq, Hkv, d, t, m = spec
    Q, K, V = make(S, beams, Hq, Hkv, d, t, m, dtype, 10)
    desc = rk.make_cross(S, beams, Hq, Hkv, d, m, rk.F32 if dtype == torch.float32 else rk.BF16)
    lengths = dev_i32([m - 7 * i for i in range(S)])
    ws = torch.empty(handle.cross_workspace_bytes(desc, t), dtype=torch.uint8, device="cuda")

    def outputs():
        return torch.empty(S * beams, Hq, t, d, dtype=dtype, device="cuda"), torch.empty(S * beams, Hq, t, device="cuda")

    want, got = outputs(), outputs()
    handle.cross_attend(desc, t, Q, K, V, want[0], ws, lengths=lengths, lse=want[1])
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    for _ in range(3):
        handle.cross_attend(desc, t, Q, K, V, got[0], ws, lengths=lengths, lse=got[1], stream=stream)
        stream.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        handle.cross_attend(desc, t, Q, K, V, got[0], ws, lengths=lengths, lse=got[1])
    lengths.copy_(dev_i32([max(0, m // 2 - 31 * i) for i in range(S)]))
    graph.replay()
    handle.cross_attend(desc, t, Q, K, V, want[0], ws, lengths=lengths, lse=want[1])
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # without the log-sum-exps the outputs are the same
    out = torch.empty_like(want[0])
    handle.cross_attend(desc, t, Q, K, V, out, ws, lengths=lengths)
    torch.cuda.synchronize()
    assert torch.equal(out, want[0])
    assert handle.poll_status() == rk.RESTKV_OK


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("spec", [(2, 3, 8, 2, 128, 1, 300), (1, 1, 4, 1, 128, 130, 257), (2, 5, 4, 4, 64, 1, 2000), (1, 2, 4, 2, 64, 100, 90), (1, 2, 3, 1, 72, 9, 40)])
def test_no_cross_write_lands_outside_a_buffer(handle, dtype, spec):
    """Outputs and workspace out of one allocation with bands of a pattern between them, which are intact afterwards."""
    S, beams, Hq, Hkv, d, t, m = spec
    b, size = S * beams, 4 if dtype == torch.float32 else 2
    Q, K, V = make(S, beams, Hq, Hkv, d, t, m, dtype, 11)
    desc = rk.make_cross(S, beams, Hq, Hkv, d, m, rk.F32 if dtype == torch.float32 else rk.BF16)
    parts = {"out": b * Hq * t * d * size, "lse": b * Hq * t * 4, "ws": handle.cross_workspace_bytes(desc, t)}
    at, total = {}, 4096
    for k, n in parts.items():
        at[k] = total
        total = -(-(total + n) // 256) * 256 + 4096
    memory = torch.full((total,), 0xA5, dtype=torch.uint8, device="cuda")
    part = {k: memory[at[k]: at[k] + n] for k, n in parts.items()}
    inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    for k, n in parts.items():
        inside[at[k]: at[k] + n] = True
    handle.cross_attend(desc, t, Q, K, V, part["out"], part["ws"], lengths=dev_i32([m - 5 * i for i in range(S)]), lse=part["lse"].view(torch.float32))
    torch.cuda.synchronize()
    assert handle.poll_status() == rk.RESTKV_OK
    assert bool((memory[~inside] == 0xA5).all())
    assert bool(torch.isfinite(part["out"].view(dtype).float()).all()) and bool(torch.isfinite(part["lse"].view(torch.float32)).all())


@pytest.mark.gpu
def test_cross_offsets_past_32_bits(handle):
    """Rows that lie more than 2^32 bytes from the first are seen where they are."""
    S, H, d, m = 3, 2, 128, 300
    gap = (1 << 31) // 2 + 1024 * d                       # elements between sources, 2 GB and some
    memory = torch.empty(2 * gap + H * m * d, dtype=torch.bfloat16, device="cuda")
    K = memory.as_strided((S, H, m, d), (gap, m * d, d, 1))
    g = torch.Generator("cuda").manual_seed(2)
    K.copy_(torch.randn(S, H, m, d, generator=g, device="cuda"))
    V = torch.randn(S, H, m, d, generator=g, device="cuda").to(torch.bfloat16)
    for t in (1, 100):
        Q = torch.randn(S, 4, t, d, generator=g, device="cuda").to(torch.bfloat16)
        check(handle, Q, K, V)


@pytest.mark.gpu
@pytest.mark.parametrize("t", [1, 6, 200])
def test_cross_in_fp32_throughout_and_where_the_tensor_cores_are_required(handle, t):
    Q, K, V = make(2, 2, 8, 2, 128, t, 333, torch.bfloat16, 12)
    try:
        handle.set_kernel_path(rk.PATH_SIMT)
        check(handle, Q, K, V, closely=True)
        handle.set_kernel_path(rk.PATH_TENSOR_CORE)
        for bad in [make(1, 1, 2, 2, 96, t, 50, torch.bfloat16, 0), make(1, 1, 2, 2, 128, t, 50, torch.float32, 0)]:
            desc = rk.make_cross(1, 1, 2, 2, bad[0].shape[3], 50, rk.F32 if bad[0].dtype == torch.float32 else rk.BF16)
            ws = torch.empty(handle.cross_workspace_bytes(desc, t), dtype=torch.uint8, device="cuda")
            with pytest.raises(rk.RestKVError) as e:
                handle.cross_attend(desc, t, *bad, torch.empty_like(bad[0]).contiguous(), ws)
            assert e.value.status == rk.ERR_UNSUPPORTED
    finally:
        handle.set_kernel_path(rk.PATH_AUTO)


# sources, beams, query heads, KV heads, head_dim, tokens, rows
SHARED = [(1, 1, 32, 8, 128, 9, 9000), (1, 3, 16, 16, 64, 11, 5000), (1, 1, 12, 4, 128, 11, 30000), (1, 33, 8, 8, 64, 1, 12345), (4, 2, 12, 4, 128, 11, 1200), (8, 1, 32, 8, 128, 10, 600),
          (1, 1, 8, 2, 128, 60, 20000), (2, 1, 4, 4, 64, 256, 4100), (2, 1, 4, 4, 128, 257, 4100), (1, 1, 3, 1, 64, 43, 40000), (5, 7, 4, 2, 128, 17, 2000), (1, 1, 1, 1, 64, 33, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("spec", SHARED)
def test_cross_units_shared_by_few_and_many_ctas(handle, spec):
    S, beams, Hq, Hkv, d, t, m = spec
    Q, K, V = make(S, beams, Hq, Hkv, d, t, m, torch.bfloat16, 15, 1.5)
    try:
        handle.set_kernel_path(rk.PATH_TENSOR_CORE)
        check(handle, Q, K, V)
        check(handle, Q, K, V, [m - m // (3 + i) * (i > 0) for i in range(S)], [(5 * i + t) % (t + 1) if i else t for i in range(S * beams)])
    finally:
        handle.set_kernel_path(rk.PATH_AUTO)


@pytest.mark.gpu
@pytest.mark.parametrize("d,t,most", [(128, 300, 1500), (64, 150, 700), (128, 1, 4000), (64, 6, 9000), (128, 40, 500)])
@pytest.mark.parametrize("kept", [0, 1, 3, 20])
def test_cross_of_sources_that_are_mostly_empty(handle, d, t, most, kept):
    """30 sources, of which some have rows, and sequences without tokens: units without work ahead of, between and behind those with it."""
    r = np.random.default_rng(100 * kept + t)
    lengths, counts = np.zeros((30, 2), int), np.zeros(60, int)
    for i in r.choice(30, kept, replace=False):
        lengths[i] = r.integers(0, most + 1, 2)
        counts[2 * i:2 * i + 2] = r.choice([0, 1, t // 2, t], 2)
    Q, K, V = make(30, 2, 4, 2, d, t, most, torch.bfloat16, 16, 1.0)
    check(handle, Q, K, V, lengths, counts)
    check(handle, Q, K, V, lengths[:, 0], counts)


@pytest.mark.gpu
@pytest.mark.parametrize("spec", [(1, 4, 8, 2, 128, 1, 1000), (2, 8, 4, 4, 64, 1, 3000), (1, 4, 32, 8, 128, 1, 40000), (1, 2, 8, 1, 64, 2, 20000), (3, 1, 4, 4, 128, 30, 700)])
def test_cross_weights_of_few_query_rows_have_two_parts(handle, spec):
    S, beams, Hq, Hkv, d, t, m = spec
    Q, K, V = make(S, beams, Hq, Hkv, d, t, m, torch.bfloat16, 17, 2.0)
    V.abs_()                                     # nothing cancels: the output's rounding and the weights' are all there is
    check(handle, Q, K, V, closely=True)


@pytest.mark.gpu
@pytest.mark.parametrize("S,beams,Hq,Hkv,d,t,m", [(1, 4, 32, 8, 128, 1, 3000), (1, 4, 32, 8, 128, 1, 40000), (1, 1, 8, 2, 128, 300, 3001), (3, 1, 8, 2, 64, 500, 700), (1, 8, 8, 2, 64, 1, 9000)])
def test_cross_waits_that_run_out(handle, S, beams, Hq, Hkv, d, t, m):
    """A wait limit of one SM clock in the tensor-core kernels of few query rows (in clusters, dealt out) and of many: whichever waits run out, the
    call returns by itself, with the timeout status or with its results, and the next one has them."""
    Q, K, V = make(S, beams, Hq, Hkv, d, t, m, torch.bfloat16, 14)
    desc = rk.make_cross(S, beams, Hq, Hkv, d, m)
    ws = torch.empty(handle.cross_workspace_bytes(desc, t), dtype=torch.uint8, device="cuda")
    lengths = dev_i32([m - 100 * i for i in range(S)])

    def call():
        out, lse = torch.empty(S * beams, Hq, t, d, dtype=torch.bfloat16, device="cuda"), torch.empty(S * beams, Hq, t, device="cuda")
        handle.cross_attend(desc, t, Q, K, V, out, ws, lengths=lengths, lse=lse)
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


# in clusters, dealt out, many query rows of either head_dim
@pytest.mark.gpu
@pytest.mark.parametrize("S,beams,Hq,Hkv,d,t,m", [(1, 4, 32, 8, 128, 1, 8000), (1, 4, 32, 8, 128, 1, 40000), (1, 1, 8, 2, 128, 300, 3001), (3, 1, 8, 2, 64, 500, 700)])
def test_cross_waits_run_out_indeed(handle, S, beams, Hq, Hkv, d, t, m):
    """With K and V in none of the caches a wait limit of one SM clock does run out, in every kernel that waits: the call returns by itself and says so, and
    the next one has its results."""
    Q, K, V = make(S, beams, Hq, Hkv, d, t, m, torch.bfloat16, 20)
    desc = rk.make_cross(S, beams, Hq, Hkv, d, m)
    ws = torch.empty(handle.cross_workspace_bytes(desc, t), dtype=torch.uint8, device="cuda")
    cold = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")

    def call():
        out, lse = torch.empty(S * beams, Hq, t, d, dtype=torch.bfloat16, device="cuda"), torch.empty(S * beams, Hq, t, device="cuda")
        cold.fill_(1)
        handle.cross_attend(desc, t, Q, K, V, out, ws, lse=lse)
        torch.cuda.synchronize()
        return handle.poll_status(), out, lse

    status, want, want_lse = call()
    assert status == rk.RESTKV_OK
    seen = []
    for _ in range(5):
        try:
            handle.set_wait_limit(1)
            seen.append(call()[0])
        finally:
            handle.set_wait_limit(2_000_000_000)
        status, out, lse = call()
        assert status == rk.RESTKV_OK and torch.equal(out, want) and torch.equal(lse, want_lse)
    assert set(seen) <= {rk.RESTKV_OK, rk.ERR_TIMEOUT} and rk.ERR_TIMEOUT in seen


STUBS = {"cross_many": """
cudaError_t cross_many_init() { return cudaFuncSetAttribute((const void*)nullptr, cudaFuncAttributeMaxDynamicSharedMemorySize, 1); }
bool cross_many_supported(const CrossProblem&) { return true; }
double cross_many_us(const CrossProblem&, int) { return 0.0; }
size_t cross_many_bytes(const CrossProblem&, int) { return 0; }
cudaError_t launch_cross_many(void*, const CrossProblem&, float*, int, long long, unsigned int*, cudaStream_t) { return cudaErrorUnknown; }
""", "cross_few": """
cudaError_t cross_few_init() { return cudaFuncSetAttribute((const void*)nullptr, cudaFuncAttributeMaxDynamicSharedMemorySize, 1); }
bool cross_few_supported(const CrossProblem&) { return true; }
double cross_few_us(const CrossProblem&, const int*) { return 0.0; }
size_t cross_few_bytes(const CrossProblem&, int) { return 0; }
cudaError_t launch_cross_few(void*, const CrossProblem&, float*, int, const int*, long long, unsigned int*, cudaStream_t, int*) { return cudaErrorUnknown; }
"""}

WITHOUT_IT = """
import sys
import torch
from paper_2605_08840_b200 import binding as rk
rk.LIB_PATH = sys.argv[1]
import test_cross as here
from helpers import DeviceRun
from paper_2605_08840_b200.inputs import Case, make_inputs
handle = rk.Handle()
run = DeviceRun(handle, make_inputs(Case("here", 1, 8, 2, 128, 2000, 32, 100, 5, 0, 0.9, "bf16", 0, "normal", 1)))
run.indices.zero_()
handle.compact(run.shape, run.K, run.V, run.indices, run.indices.shape[2], run.K_out, run.V_out)      # no launch finds an error of the handle's creation
handle.set_kernel_path(rk.PATH_TENSOR_CORE)
run.evict()
assert handle.poll_status() == rk.RESTKV_OK
refused = 0
for path in (rk.PATH_TENSOR_CORE, rk.PATH_AUTO):
    handle.set_kernel_path(path)
    for t in (1, 200):
        try:
            here.check(handle, *here.make(2, 2, 8, 2, 128, t, 333, torch.bfloat16, 1))
        except rk.RestKVError as e:
            assert e.status == rk.ERR_UNSUPPORTED and path == rk.PATH_TENSOR_CORE, e
            refused += 1
print("refused", refused)
"""


@pytest.mark.gpu
@pytest.mark.parametrize("name,refused", [("cross_many", 0), ("cross_few", 1)])
def test_a_kernel_that_cannot_run_takes_no_other_with_it(tmp_path, name, refused):
    """A library in which one of the tensor-core kernels of the cross attention finds at the handle's creation that it cannot run: scores are made on the
    tensor cores all the same, and cross attention by the kernels that are left."""
    stub, obj, lib = tmp_path / "stub.cu", tmp_path / "stub.o", tmp_path / "without.so"
    stub.write_text('#include "cross.cuh"\nnamespace restkv {\n%s\n}\n' % STUBS[name])
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc] + rk_build.COMPILE_FLAGS + ["-I", rk_build.CSRC, "-o", str(obj), str(stub)], check=True, capture_output=True)
    os.makedirs(rk_build.OBJ, exist_ok=True)
    objs = []
    for source in rk_build.sources():
        made = os.path.join(rk_build.OBJ, os.path.basename(source)[:-3] + ".o")
        if os.path.basename(made) == name + ".o":
            made = str(obj)
        elif not os.path.exists(made):          # (a library may have come without what it was linked from)
            subprocess.run([nvcc] + rk_build.COMPILE_FLAGS + ["-o", made, source], check=True, capture_output=True)
        objs.append(made)
    subprocess.run([nvcc] + rk_build.LINK_FLAGS + ["-o", str(lib)] + objs, check=True, capture_output=True)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([root, os.path.join(root, "tests")]))
    res = subprocess.run([sys.executable, "-c", WITHOUT_IT, str(lib)], cwd=root, env=env, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
    assert res.stdout.split() == ["refused", str(refused)]


# ---- refusals -------------------------------------------------------------------------------------------------------------------------

def good(**kw):
    a = dict(sources=2, beams=3, n_q_heads=8, n_kv_heads=2, head_dim=128, n_rows=100)
    a.update(kw)
    return rk.make_cross(**a)


REFUSED = [(dict(sources=0), 1), (dict(beams=0), 1), (dict(n_q_heads=7), 1), (dict(n_kv_heads=0), 1), (dict(head_dim=0), 1), (dict(n_rows=0), 1), (dict(dtype=5), 1),
           (dict(lengths_per_head=2), 1), (dict(softmax_scale=-1.0), 1), (dict(softmax_scale=float("nan")), 1), (dict(softmax_scale=float("inf")), 1), (dict(head_dim=100), 2),
           (dict(head_dim=264), 2), (dict(sources=40000), 2), (dict(n_rows=2 ** 31 - 1), 2), (dict(beams=2 ** 30), 2)]


@pytest.mark.parametrize("change,status", REFUSED)
def test_sizes_of_refused_cross_attention_are_zero(change, status):
    lib = rk.load_library()
    assert lib.restkv_cross_workspace_bytes(ctypes.byref(good()), 1) > 0
    assert lib.restkv_cross_workspace_bytes(ctypes.byref(good(**change)), 1) == 0
    assert lib.restkv_cross_workspace_bytes(ctypes.byref(good()), 0) == 0
    assert lib.restkv_cross_workspace_bytes(None, 1) == 0


def test_null_handle_is_rejected():
    assert rk.load_library().restkv_cross_attend(None, ctypes.byref(good()), 1, None, None, None, None, None, None, None, None, 0, None) == rk.ERR_INVALID_ARG


@pytest.mark.parametrize("dtype", [rk.BF16, rk.F32])
@pytest.mark.parametrize("S,beams,Hq,Hkv,d", [(1, 1, 32, 8, 128), (1, 4, 8, 8, 64), (3, 5, 6, 2, 96), (8, 1, 16, 1, 256), (70, 2, 4, 4, 128), (1, 1, 1, 1, 8)])
@pytest.mark.parametrize("m", [1, 100, 100000])
def test_workspaces_serve_calls_of_fewer_tokens(dtype, S, beams, Hq, Hkv, d, m):
    lib = rk.load_library()
    desc = rk.make_cross(S, beams, Hq, Hkv, d, m, dtype)
    sizes = [lib.restkv_cross_workspace_bytes(ctypes.byref(desc), t) for t in (1, 2, 3, 5, 8, 16, 17, 31, 33, 64, 65, 100, 129, 300, 1000, 5000)]
    assert sizes == sorted(sizes) and sizes[0] > 0 and all(n % 256 == 0 for n in sizes)


@pytest.mark.gpu
def test_cross_refusals_enqueue_nothing(handle):
    Q, K, V = make(2, 3, 8, 2, 128, 2, 100, torch.bfloat16, 0)
    out, lengths = torch.zeros(6, 8, 2, 128, dtype=torch.bfloat16, device="cuda"), dev_i32([100, 100])
    ws = torch.empty(handle.cross_workspace_bytes(good(), 2) + 256, dtype=torch.uint8, device="cuda")
    before = handle.launch_count()

    def refused(status, desc=None, t=2, Q=Q, K=K, V=V, out=out, ws=ws, lengths=lengths):
        with pytest.raises(rk.RestKVError) as e:
            handle.cross_attend(desc or good(), t, Q, K, V, out, ws, lengths=lengths)
        assert e.value.status == status

    for change, status in REFUSED:
        refused(status, desc=good(**change))
    refused(rk.ERR_INVALID_ARG, t=0)
    refused(rk.ERR_INVALID_ARG, out=None)
    refused(rk.ERR_INVALID_ARG, out=out.view(-1)[4:])
    refused(rk.ERR_INVALID_ARG, desc=good(lengths_per_head=1), lengths=None)
    flat = torch.zeros(1 << 20, dtype=torch.bfloat16, device="cuda")
    refused(rk.ERR_INVALID_ARG, K=flat[4:].as_strided((2, 2, 100, 128), (25600, 12800, 128, 1)))
    refused(rk.ERR_INVALID_ARG, V=flat.as_strided((2, 2, 100, 128), (25600, 12804, 128, 1)))
    refused(rk.ERR_WORKSPACE, ws=ws[16:])
    refused(rk.ERR_WORKSPACE, ws=ws[: handle.cross_workspace_bytes(good(), 2) - 256])
    assert handle.launch_count() == before
    # the strides of dimensions of one are not looked at
    one = flat.as_strided((1, 1, 1, 128), (4, 12, 20, 1))
    desc = rk.make_cross(1, 1, 1, 1, 128, 1)
    handle.cross_attend(desc, 1, one, one, one, out.view(-1)[:128], torch.empty(handle.cross_workspace_bytes(desc, 1), dtype=torch.uint8, device="cuda"))
    assert handle.poll_status() == rk.RESTKV_OK


# ---- what it is used with ---------------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("per_head", [False, True])
def test_an_encoder_s_states_are_evicted_by_what_the_decoder_s_prompt_saw(handle, per_head):
    """A decoder prompt attends to an encoder's rows; its last 32 tokens' outputs and log-sum-exps are what the eviction takes; tokens of four
    hypotheses then attend to the rows that were kept, of every head as many as its budget lets it keep."""
    Hq, Hkv, d, m, w, budget, t, beams = 32, 8, 128, 3000, 32, 400, 70, 4
    Q, K, V = make(1, 1, Hq, Hkv, d, t, m, torch.bfloat16, 13, 1.0, "dense")
    K[:, :, 1000:1040] += 0.5 * Q[:, ::4, -1:, :]          # rows that the last token sees
    out, lse = check(handle, Q, K, V)
    shape = rk.make_shape(1, Hq, Hkv, d, m, w)
    window = Q[:, :, -w:].contiguous()
    Ko, Vo = (torch.zeros(1, Hkv, budget, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    indices, scores, want = dev_i32(np.zeros((1, Hkv, budget))), torch.empty(1, Hkv, m, device="cuda"), torch.empty(1, Hkv, m, device="cuda")
    ws = torch.empty(handle.workspace_bytes(shape, budget), dtype=torch.uint8, device="cuda")
    handle.evict_from_lse(shape, window, K, V, out[:, :, -w:].float().contiguous(), lse[:, :, -w:].contiguous(), 0.9, rk.fixed_pool(7), budget, indices, Ko, Vo, ws, scores_out=scores)
    handle.score(shape, window, K, V, 0.9, rk.fixed_pool(7), want, ws)
    torch.cuda.synchronize()
    assert bool(((scores - want).abs() <= 4e-3 * want.abs()).all())      # both within 2e-3 of the formula
    lengths = [budget]
    if per_head:
        lengths = [[budget - 40 * h for h in range(Hkv)]]
        handle.evict_budgets(shape, window, K, V, 0.9, rk.fixed_pool(7), dev_i32(lengths), budget, indices, Ko, Vo, ws)
    kept = indices.long().clamp(min=0)[..., None].expand(1, Hkv, budget, d)
    token = torch.randn(beams, Hq, 1, d, device="cuda").to(torch.bfloat16)
    check(handle, token, Ko, Vo, lengths)
    for x, y in ((K, Ko), (V, Vo)):
        for h in range(Hkv):
            n = lengths[0][h] if per_head else budget
            assert torch.equal(x.gather(2, kept)[0, h, :n], y[0, h, :n])
