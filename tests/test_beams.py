"""Decoding with beams: the best continuations of every request's hypotheses, the paged cache brought in the order of their parents, against plain
implementations in 64 bits that are written from the header's definitions."""
import ctypes
import subprocess

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


# ---- selection ------------------------------------------------------------------------------------------------------------------------

class Plain:
    """The continuations of one request in 64 bits."""

    def __init__(self, logits, scores, finished, n_out, pad):
        self.beams, self.vocab = logits.shape
        x = logits.astype(np.float64)
        self.x = np.where(np.isnan(x), NEG_INF, np.minimum(x, float(np.finfo(np.float32).max)))
        self.scores = [NEG_INF if np.isnan(s) else float(s) for s in scores]
        self.finished, self.pad = finished if finished is not None else [0] * self.beams, pad
        top = self.x.max(1)
        with np.errstate(divide="ignore", invalid="ignore"):
            self.total = np.where(top > NEG_INF, top + np.log(np.exp(self.x - top[:, None]).sum(1)), 0.0)
        rows = []
        for k in range(self.beams):
            if self.finished[k]:
                rows.append((k, pad, 0.0))
            elif self.scores[k] == NEG_INF:
                rows += [(k, v, 0.0) for v in range(min(n_out, self.vocab))]
            else:
                rows += [(k, int(v), self.x[k, v]) for v in np.lexsort((np.arange(self.vocab), -self.x[k]))[:n_out]]
        rows.sort(key=lambda r: (-self.score(*r[:2]), r[0], -r[2], r[1]))
        self.best = [r[:2] for r in rows[:n_out]]

    def score(self, k, v):
        if self.finished[k]:
            return self.scores[k] if v == self.pad else np.nan
        if self.scores[k] == NEG_INF or self.x[k, v] == NEG_INF:
            return NEG_INF
        return self.scores[k] + (self.x[k, v] - self.total[k])


# The normaliser is off by at most: 2^-22 of an exponential's own, 2^-24 each for a difference and its product with log2 e, which weigh |arg| 2^-|arg|
# (their sum over the terms at most 24 |arg| units below 2^-24 of the largest), some 31 fp32 additions of 2^-24, twice the exponentials that join
# slices and warps.  The score comes out rounded to fp32.
def select_slack(score):
    return 2.0 ** -22 + 2 * 24 * 0.7 * 2.0 ** -24 + 31 * 2.0 ** -24 + 2 * 2.0 ** -22 + 2.0 ** -24 * abs(score)


def check_select(handle, logits, scores, n_out, finished=None, pad=3, stride_pad=0, exact_ties=False):
    """logits: a tensor [batch, beams, vocab] on the device."""
    batch, beams, vocab = logits.shape
    dtype = rk.F32 if logits.dtype == torch.float32 else rk.BF16
    held = torch.full((batch * beams, vocab + stride_pad), float("nan"), dtype=logits.dtype, device="cuda")
    held[:, :vocab] = logits.reshape(-1, vocab)
    desc = rk.make_beams(batch, beams, vocab, n_out, dtype, vocab + stride_pad, pad)
    ws = torch.full((handle.beam_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda")
    parents, tokens = (torch.full((batch, n_out), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    out = torch.full((batch, n_out), float("nan"), device="cuda")
    scores = torch.as_tensor(scores, dtype=torch.float32).cuda()
    done = None if finished is None else torch.as_tensor(np.asarray(finished).astype(np.uint8)).cuda()
    handle.beam_select(desc, held, scores, parents, tokens, out, ws, finished=done)
    torch.cuda.synchronize()
    assert handle.poll_status() == rk.RESTKV_OK
    x, s = logits.float().cpu().numpy(), scores.cpu().numpy()
    for b in range(batch):
        plain = Plain(x[b], s[b], None if finished is None else np.asarray(finished)[b], n_out, pad)
        got = list(zip(parents[b].tolist(), tokens[b].tolist()))
        for i, (k, v) in enumerate(got):
            score = float(out[b, i])
            if i >= len(plain.best):
                assert (k, v, score) == (0, pad, NEG_INF)
                continue
            exact, want = plain.score(k, v), plain.score(*plain.best[i])
            if np.isinf(want) or np.isinf(exact) or exact_ties:
                assert (k, v) == plain.best[i], (b, i, k, v, plain.best[i])
                if np.isinf(want):
                    assert score == want
                    continue
            slack = select_slack(want)
            assert abs(score - exact) <= slack, (b, i, score, exact)
            # in the place of another only where what is off may have brought it there
            assert (k, v) == plain.best[i] or (abs(exact - want) <= 2 * slack and plain.best[i][0] != k), (b, i, k, v, plain.best[i])
        assert len(set(got[: len(plain.best)])) == len(plain.best)
    return parents, tokens, out


SELECT = [(1, 1, 1, 1), (1, 1, 5, 5), (1, 2, 3, 6), (2, 3, 2, 20), (3, 4, 1000, 8), (2, 5, 4099, 10), (1, 4, 32000, 8), (2, 3, 16384, 6), (1, 2, 16385, 4), (4, 2, 50257, 4),
          (1, 16, 8191, 32), (2, 64, 257, 64), (1, 1, 131072, 64), (40, 8, 9000, 16), (1, 3, 300001, 6)]


@pytest.mark.gpu
@pytest.mark.parametrize("spec", SELECT)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("stride_pad", [0, 3])
def test_select(handle, spec, dtype, stride_pad):
    batch, beams, vocab, n_out = spec
    rng = np.random.default_rng(sum(spec) + stride_pad)
    logits = torch.from_numpy((rng.standard_normal((batch, beams, vocab)) * 3).astype(np.float32)).cuda().to(dtype)
    check_select(handle, logits, -10 * rng.random((batch, beams)), n_out, stride_pad=stride_pad)


@pytest.mark.gpu
@pytest.mark.parametrize("spec", [(1, 64, 20000, 64), (2, 33, 9001, 40), (3, 16, 4096, 64), (1, 1, 262144, 64), (2, 64, 4096, 63)])
@pytest.mark.parametrize("spread", [0.0, 1.0, 30.0])
def test_select_many_of_many(handle, spec, spread):
    """More candidates than a block holds at a time, hypotheses of like scores and of such that one of them has nearly all."""
    batch, beams, vocab, n_out = spec
    rng = np.random.default_rng(vocab + int(spread))
    logits = torch.from_numpy((rng.standard_normal((batch, beams, vocab)) * 2).astype(np.float32)).cuda().bfloat16()
    finished = np.zeros((batch, beams), bool)
    if beams > 2:
        finished[:, 2::7] = True
    check_select(handle, logits, -spread * rng.random((batch, beams)), n_out, finished)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab,n_out", [(777, 12), (20001, 8), (40, 64)])
def test_select_with_ended_and_absent_hypotheses(handle, dtype, vocab, n_out):
    rng = np.random.default_rng(vocab)
    batch, beams = 7, 6
    logits = torch.from_numpy(rng.standard_normal((batch, beams, vocab)).astype(np.float32)).cuda().to(dtype)
    logits[:, :, ::3] = NEG_INF
    scores = -3 * rng.random((batch, beams))
    finished = rng.random((batch, beams)) < 0.4
    finished[0] = True                          # all have ended
    finished[1], scores[1, 1:] = False, NEG_INF  # the first step
    scores[2] = NEG_INF                         # nothing there at all
    finished[2] = [0, 1, 0, 1, 1, 0]
    scores[3, 2] = np.nan
    finished[3, 2] = False
    scores[3, 4] = np.nan
    finished[3, 4] = True
    finished[4] = [0, 1, 1, 1, 1, 1]
    logits[4, 0] = NEG_INF                      # the only one that goes on may not by any token
    logits[5, :, 5:] = NEG_INF                  # a handful of tokens is allowed
    finished[6] = False
    check_select(handle, logits, scores, n_out, finished)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [1000, 50257, 70000])
@pytest.mark.parametrize("n_out", [4, 64])
def test_select_ties(handle, dtype, vocab, n_out):
    """Equal logits, equal rows, equal requests: the lower hypothesis, then the lower token, exactly."""
    beams = 3
    flat = torch.zeros(2, beams, vocab, dtype=dtype, device="cuda")
    flat[1] = -2.0
    flat[1, :, -1] = 2.0 ** -20                 # one that stands out, the last token
    check_select(handle, flat, np.zeros((2, beams)), n_out, exact_ties=True)
    # rows that begin at different places of their first 16 bytes are equal all the same
    rng = np.random.default_rng(n_out)
    one = torch.from_numpy(rng.standard_normal(vocab).astype(np.float32)).cuda().to(dtype)
    check_select(handle, one.expand(2, beams, vocab), np.full((2, beams), -1.25), n_out, exact_ties=True)
    few = torch.from_numpy(rng.integers(-3, 3, vocab).astype(np.float32)).cuda().to(dtype)
    check_select(handle, few.expand(1, beams, vocab), np.zeros((1, beams)), n_out, stride_pad=1, exact_ties=True)
    # and -0 is 0
    signs = torch.where(torch.arange(vocab, device="cuda") % 2 == 0, -0.0, 0.0).to(dtype)
    check_select(handle, signs.expand(1, 1, vocab), np.zeros((1, 1)), n_out, exact_ties=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("batch,vocab", [(1, 9000), (40, 30000)])
@pytest.mark.parametrize("low", [False, True])
def test_select_of_more_equal_logits_than_a_list_holds_every_time(handle, dtype, batch, vocab, low):
    """Slices of more than 2048 equal logits (the bound is found anew among logits with their tokens), and of such that one group of threads has only
    lower ones (so that this bound holds back nothing either), call after call: the same continuations, by the order that the header states."""
    beams, n_out = 3, 64
    at = torch.arange(vocab, device="cuda") // (16 // torch.empty(0, dtype=dtype).element_size()) % 256
    x = torch.where(at < 4, 0.0, 1.0).to(dtype) if low else torch.ones(vocab, dtype=dtype, device="cuda")
    logits = x.expand(batch, beams, vocab)
    want = check_select(handle, logits, np.zeros((batch, beams)), n_out, exact_ties=True)
    desc = rk.make_beams(batch, beams, vocab, n_out, rk.F32 if dtype == torch.float32 else rk.BF16)
    held, scores = logits.reshape(-1, vocab).contiguous(), torch.zeros(batch, beams, device="cuda")
    ws = torch.empty(handle.beam_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    for _ in range(50):
        got = [torch.full_like(x, -7) for x in want]
        handle.beam_select(desc, held, scores, *got, ws)
        assert all(torch.equal(x, y) for x, y in zip(want, got))
    assert handle.poll_status() == rk.RESTKV_OK


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("order", ["up", "down", "strided", "steps"])
def test_select_where_the_largest_lie_close_together(handle, dtype, order):
    vocab = 33000
    x = np.linspace(-20, 20, vocab)
    if order == "down":
        x = x[::-1]
    elif order == "strided":                    # the largest all with the same threads
        x = np.where(np.arange(vocab) % 2048 < 8, x, -30)
    elif order == "steps":
        x = np.floor(x / 4)
    logits = torch.from_numpy(np.ascontiguousarray(np.stack([x, x[::-1]])[None], np.float32)).cuda().to(dtype)
    for n_out in (1, 7, 64):
        check_select(handle, logits, [[-1.0, -1.5]], n_out)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_select_what_no_model_should_make(handle, dtype):
    """NaN counts as -inf and +inf as the largest number, wherever they stand; logits of any size."""
    rng = np.random.default_rng(5)
    x = rng.standard_normal((6, 2, 5003)).astype(np.float32)
    x[0, 0, rng.integers(0, 5003, 40)] = np.nan
    x[0, 1, 17] = np.inf
    x[1, 0] = np.nan
    x[1, 1, :5000] = -np.inf
    x[2, 0, 100:110] = np.inf
    x[2, 1, 7], x[2, 1, 8] = np.nan, np.inf
    x[3] *= 1e30
    x[4] *= 1e-30
    x[5, 0], x[5, 1] = -3.3e38, 3.3e38
    check_select(handle, torch.from_numpy(x).cuda().to(dtype), -rng.random((6, 2)), 9)
    scores = np.array([[np.inf, 0.0], [-np.inf, 1e30], [-1e38, -1.0], [0.0, -0.0], [5.0, np.nan], [0.0, 0.0]])
    check_select(handle, torch.from_numpy(x).cuda().to(dtype), scores, 9)


@pytest.mark.gpu
def test_select_same_bits_in_a_graph_on_another_stream_and_over_its_scores(handle):
    g = torch.Generator("cuda").manual_seed(3)
    logits = torch.randn(24, 20011, generator=g, device="cuda")
    scores = -torch.rand(4, 6, generator=g, device="cuda")
    desc = rk.make_beams(4, 6, 20011, 6, rk.F32)
    ws = torch.empty(handle.beam_workspace_bytes(desc), dtype=torch.uint8, device="cuda")

    def outputs():
        return [torch.empty(4, 6, dtype=torch.int32, device="cuda"), torch.empty(4, 6, dtype=torch.int32, device="cuda"), torch.empty(4, 6, device="cuda")]

    want, got = outputs(), outputs()
    handle.beam_select(desc, logits, scores, *want, ws)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    handle.beam_select(desc, logits, scores, *got, ws, stream=stream)
    stream.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        handle.beam_select(desc, logits, scores, *got, ws)
    logits.copy_(torch.randn(24, 20011, generator=g, device="cuda"))
    graph.replay()
    handle.beam_select(desc, logits, scores, *want, ws)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    handle.beam_select(desc, logits, scores, got[0], got[1], scores, ws)      # the scores are brought up to date in place
    torch.cuda.synchronize()
    assert torch.equal(scores, want[2]) and torch.equal(got[1], want[1])


def test_nothing_behind_the_rows_of_logits_is_read(tmp_path):
    """The 16-byte pieces that are loaded of rows of any length and stride: none reaches behind the last row's end; what is taken from them lies in pieces that
    are loaded; and no more than two runs of 16 bytes of a row are left, which are loaded token by token."""
    source = tmp_path / "pieces.cc"
    source.write_text("""
#include <cstdio>
#include <initializer_list>
#include "row_pieces.cuh"
template <bool kRagged> void print(int off, int n, int size) {
  const restkv::RowPieces<kRagged> r((unsigned int)off, n, size);
  std::printf(" %d %d", r.loaded, r.inside);
}
int main() {
  for (int size : {2, 4})
    for (int n : {1, 2, 3, 4, 5, 6, 7, 8, 9, 15, 16, 17, 31, 100, 257, 50257, 131072, 0x40000000})
      for (int pad : {0, 1, 2, 3, 5, 8})
        for (int rows : {1, 2, 3, 4, 8, 81}) {
          const bool ragged = restkv::rows_end_inside_a_piece(rows, (long long)n + pad, n, size);
          for (int row = 0; row < rows; ++row) {
            std::printf("%d %d %d %d %d %d", size, n, pad, rows, row, (int)ragged);
            const int off = (int)(row * ((long long)n + pad) * size % 16);
            ragged ? print<true>(off, n, size) : print<false>(off, n, size);
            std::printf("\\n");
          }
        }
}
""")
    program = tmp_path / "pieces"
    subprocess.run(["g++", "-std=c++17", "-I", rk_build.CSRC, "-o", str(program), str(source)], check=True)
    lines = subprocess.run([str(program)], check=True, capture_output=True, text=True).stdout.split("\n")[:-1]
    assert len(lines) == 2 * 18 * 6 * (1 + 2 + 3 + 4 + 8 + 81)
    for line in lines:
        size, n, pad, rows, row, ragged, loaded, inside = (int(x) for x in line.split())
        begin = row * (n + pad) * size
        off, end, last = begin % 16, begin + n * size, ((rows - 1) * (n + pad) + n) * size
        assert begin - off + 16 * loaded <= last, line
        if ragged:                              # from piece `inside` on token by token
            assert begin + 16 * max(0, inside) <= end and (inside <= 0 or off + 16 * inside <= 16 * loaded), line
            assert -(-(end - begin) // 16) - max(0, inside) <= 2, line
        else:
            assert begin - off + 16 * loaded >= end, line


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("stride_pad", [0, 1, 5])
def test_select_by_the_last_tokens_of_rows_of_any_length(handle, dtype, stride_pad):
    """The largest logits are a row's last ones, in whatever part of 16 bytes it ends, alone in their slice or not."""
    rng = np.random.default_rng(stride_pad)
    for vocab in [*range(1, 20), *range(2040, 2060), *range(4090, 4106), 8193, 50257]:
        x = rng.standard_normal((3, 2, vocab)).astype(np.float32)
        x[:, :, -3:] = 20 + np.arange(min(3, vocab))
        x[1, 0, -1] = np.nan
        check_select(handle, torch.from_numpy(x).cuda().to(dtype), -rng.random((3, 2)), 5, stride_pad=stride_pad)


def good_beams(**kw):
    a = dict(batch=2, beams=4, vocab=1000, n_out=8)
    a.update(kw)
    return rk.make_beams(**a)


REFUSED_BEAMS = [(dict(batch=0), 1), (dict(beams=0), 1), (dict(vocab=0), 1), (dict(n_out=0), 1), (dict(dtype=2), 1), (dict(stride=999), 1), (dict(stride=-1), 1), (dict(beams=65), 2),
                 (dict(n_out=65), 2), (dict(vocab=2 ** 30 + 1), 2), (dict(batch=2 ** 30), 2)]


@pytest.mark.parametrize("change,status", REFUSED_BEAMS)
def test_sizes_of_refused_selections_are_zero(change, status):
    lib = rk.load_library()
    assert lib.restkv_beam_workspace_bytes(ctypes.byref(good_beams())) > 0
    assert lib.restkv_beam_workspace_bytes(ctypes.byref(good_beams(**change))) == 0
    assert lib.restkv_beam_workspace_bytes(None) == 0


@pytest.mark.gpu
def test_select_refusals_enqueue_nothing(handle):
    logits, scores = torch.zeros(8, 1000, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 4, device="cuda")
    parents, tokens, out = dev_i32(np.zeros((2, 8))), dev_i32(np.zeros((2, 8))), torch.zeros(2, 8, device="cuda")
    desc = good_beams()
    ws = torch.empty(handle.beam_workspace_bytes(desc) + 256, dtype=torch.uint8, device="cuda")
    before = handle.launch_count()

    def refused(status, desc=desc, logits=logits, scores=scores, parents=parents, ws=ws):
        with pytest.raises(rk.RestKVError) as e:
            handle.beam_select(desc, logits, scores, parents, tokens, out, ws)
        assert e.value.status == status

    for change, status in REFUSED_BEAMS:
        refused(status, desc=good_beams(**change))
    refused(rk.ERR_INVALID_ARG, logits=None)
    refused(rk.ERR_INVALID_ARG, scores=None)
    refused(rk.ERR_INVALID_ARG, parents=None)
    refused(rk.ERR_INVALID_ARG, logits=logits.view(-1)[1:])
    refused(rk.ERR_WORKSPACE, ws=ws[16:])
    refused(rk.ERR_WORKSPACE, ws=ws[: handle.beam_workspace_bytes(desc) - 256])
    assert handle.launch_count() == before


# ---- reordering -------------------------------------------------------------------------------------------------------------------------

def reorder_plain(table, parents, n, page_rows):
    """(new table, copies, dropped) of one request."""
    beams, full, rest = len(table), n // page_rows, n % page_rows
    free = [j for j in range(beams) if j not in parents]
    seen, new, copies = set(), [], []
    for p in parents:
        donor = free.pop(0) if p in seen else p
        seen.add(p)
        new.append(list(table[p][:full]) + list(table[donor][full:]))
        copies.append((table[p][full], table[donor][full], rest) if donor != p and rest else (-1, -1, 0))
    dropped = [[-1] * len(table[0]) for _ in table]
    for c in range(full):
        left = {table[p][c] for p in parents}
        for j in range(beams):
            if table[j][c] not in left:
                dropped[j][c] = table[j][c]
                left.add(table[j][c])
    return new, copies, dropped


def tree_tables(rng, requests, beams, full, width, spare=2):
    """Tables of hypotheses that share their first pages as the branches of a tree do, with pages of their own from column `full` on."""
    ids = iter(rng.permutation(requests * beams * width + spare).tolist())
    tables = np.empty((requests, beams, width), np.int64)
    for r in range(requests):
        for c in range(width):
            if c >= full:
                owner = list(range(beams))
            elif c == 0:
                owner = [0] * beams
            else:                               # groups that split further with every column
                owner = [int(x) for x in rng.integers(0, min(beams, c + 1), beams)] if c % 3 else [0] * beams
            page = {}
            for j in range(beams):
                if owner[j] not in page:
                    page[owner[j]] = next(ids)
                tables[r, j, c] = page[owner[j]]
    return tables


REORDER = [(1, 1, 100, 16, 8), (1, 4, 2085, 64, 33), (3, 5, 37, 16, 4), (2, 8, 512, 32, 17), (2, 8, 512, 32, 16), (4, 64, 130, 16, 10), (1, 33, 15, 16, 1), (2, 3, 0, 48, 5),
           (1, 2, 4000, 16, 300), (2, 6, 1000, 256, 130)]


@pytest.mark.gpu
@pytest.mark.parametrize("spec", REORDER)
@pytest.mark.parametrize("in_place", [False, True])
def test_reorder(handle, spec, in_place):
    requests, beams, n, R, width = spec
    rng = np.random.default_rng(sum(spec) + in_place)
    for kind in ("any", "same", "fork", "last", "turn"):
        table = tree_tables(rng, requests, beams, n // R, width)
        parents = {"any": rng.integers(0, beams, (requests, beams)), "same": np.tile(np.arange(beams), (requests, 1)), "fork": np.zeros((requests, beams), np.int64),
                   "last": np.full((requests, beams), beams - 1), "turn": np.tile(np.roll(np.arange(beams), 1), (requests, 1))}[kind]
        desc = rk.make_paged(requests * beams, 4, 2, 64, rk.PAGES_BF16, R, int(table.max()) + 3, width)
        old = dev_i32(table.reshape(-1, width))
        new = old.clone() if in_place else torch.full_like(old, -99)
        copies, dropped = torch.full((requests * beams, 3), -99, dtype=torch.int32, device="cuda"), torch.full_like(old, -99)
        handle.paged_reorder(desc, beams, dev_i32(parents), dev_i32([n] * requests * beams), new if in_place else old, new, copies, dropped=dropped)
        torch.cuda.synchronize()
        assert handle.poll_status() == rk.RESTKV_OK
        for r in range(requests):
            t, c, d = reorder_plain(table[r].tolist(), parents[r].tolist(), n, R)
            at = slice(r * beams, (r + 1) * beams)
            assert new[at].tolist() == t, kind
            assert copies[at].tolist() == [list(x) for x in c], kind
            assert dropped[at].tolist() == d, kind
        # every sequence's own page is nobody else's
        if n % R:
            own = new.view(requests, beams, width)[:, :, n // R]
            assert all(len(set(x)) == beams for x in own.tolist())


@pytest.mark.gpu
def test_reorder_leaves_requests_that_cannot_be(handle):
    beams, width, R = 4, 5, 16
    rng = np.random.default_rng(0)
    table = tree_tables(rng, 5, beams, 2, width)
    old = dev_i32(table.reshape(-1, width))
    desc = rk.make_paged(5 * beams, 4, 2, 64, rk.PAGES_BF16, R, 200, width)
    parents = np.zeros((5, beams), np.int64)
    parents[1, 2], parents[2, 0] = beams, -1
    lengths = np.full((5, beams), 40)
    lengths[3, 1] = 41
    lengths[4] = R * width + 1
    for in_place in (False, True):
        src = old.clone()
        new = src if in_place else torch.zeros_like(old)
        copies, dropped = torch.zeros(5 * beams, 3, dtype=torch.int32, device="cuda"), torch.zeros_like(old)
        handle.paged_reorder(desc, beams, dev_i32(parents), dev_i32(lengths.reshape(-1)), src, new, copies, dropped=dropped)
        assert handle.poll_status() == rk.ERR_INVALID_ARG
        assert handle.poll_status() == rk.RESTKV_OK
        t, c, d = reorder_plain(table[0].tolist(), [0] * beams, 40, R)
        assert new[:beams].tolist() == t and copies[:beams].tolist() == [list(x) for x in c] and dropped[:beams].tolist() == d
        assert torch.equal(new[beams:], old[beams:])
        assert bool((copies[beams:] == dev_i32([-1, -1, 0])).all()) and bool((dropped[beams:] == -1).all())
    # a page that has to be copied and is none
    bad = old.clone()
    bad[0, 2] = 200
    handle.paged_reorder(desc, beams, dev_i32(np.zeros((5, beams))), dev_i32([40] * 5 * beams), bad, torch.zeros_like(old), copies)
    assert handle.poll_status() == rk.ERR_INVALID_ARG


COPY = [("bf16", 64, 2, 64, 0), ("bf16", 128, 8, 16, 0), ("f32", 96, 3, 48, 0), ("int4", 128, 2, 64, 32), ("int4", 64, 1, 256, 64), ("bf16", 256, 1, 256, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("spec", COPY)
@pytest.mark.parametrize("layers,gap", [(1, 0), (3, 0), (2, 4096)])
def test_copy(handle, spec, layers, gap):
    fmt, d, H, R, group = spec
    n_pages = 9
    desc = rk.make_paged(4, H, H, d, {"bf16": rk.PAGES_BF16, "f32": rk.PAGES_F32, "int4": rk.PAGES_INT4}[fmt], R, n_pages, 2, group,
                         rk.F32 if fmt == "f32" else rk.BF16)
    page = handle.paged_page_bytes(desc)
    stride = n_pages * page + gap
    g = torch.Generator("cuda").manual_seed(R + d)
    pools = [torch.randint(0, 256, (layers * stride + 512,), generator=g, dtype=torch.uint8, device="cuda") for _ in range(2)]
    rows = [R, 1, 17, 0, R - 1]
    copies = [(0, 5, rows[0]), (1, 6, rows[1]), (1, 7, min(rows[2], R)), (2, 8, rows[3]), (-1, -1, 0), (3, 4, rows[4]), (2, 2, 5)]
    want = [p.clone() for p in pools]
    unit = R // 16 if fmt == "int4" else R
    for w in want:
        for layer in range(layers):
            x = w[layer * stride: layer * stride + n_pages * page].view(n_pages, H, unit, -1)
            for src, dst, n in copies:
                if src >= 0:
                    m = -(-n // 16) if fmt == "int4" else n
                    x[dst, :, :m] = x[src, :, :m].clone()
    handle.paged_copy(desc, dev_i32(copies), pools[0], pools[1], n_layers=layers, layer_bytes=stride if gap else 0)
    torch.cuda.synchronize()
    assert handle.poll_status() == rk.RESTKV_OK
    assert torch.equal(pools[0], want[0]) and torch.equal(pools[1], want[1])
    # what is no page, or no number of its rows, is left out
    for bad in [(n_pages, 0, 1), (0, n_pages, 1), (0, -1, 1), (0, 1, R + 1), (0, 1, -1)]:
        handle.paged_copy(desc, dev_i32([bad, (1, 6, 1)]), pools[0], pools[1], n_layers=layers, layer_bytes=stride if gap else 0)
        assert handle.poll_status() == rk.ERR_INVALID_ARG
    assert torch.equal(pools[0], want[0]) and torch.equal(pools[1], want[1])


def test_null_handle_is_rejected():
    lib = rk.load_library()
    beams, cache = good_beams(), rk.make_paged(4, 4, 2, 64, rk.PAGES_BF16, 16, 8, 2)
    assert lib.restkv_beam_select(None, ctypes.byref(beams), None, None, None, None, None, None, None, 0, None) == rk.ERR_INVALID_ARG
    assert lib.restkv_paged_reorder(None, ctypes.byref(cache), 2, None, None, None, None, None, None, None) == rk.ERR_INVALID_ARG
    assert lib.restkv_paged_copy(None, ctypes.byref(cache), None, 1, None, None, 1, 0, None) == rk.ERR_INVALID_ARG


@pytest.mark.gpu
def test_reorder_and_copy_refusals_enqueue_nothing(handle):
    def cache(**kw):
        a = dict(batch=4, n_q_heads=4, n_kv_heads=2, head_dim=64, page_format=rk.PAGES_BF16, page_rows=16, n_pages=8, table_width=2)
        a.update(kw)
        return rk.make_paged(**a)

    table, parents, lengths = dev_i32(np.zeros((9, 2))), dev_i32([0] * 4), dev_i32([5] * 4)
    copies = dev_i32(np.full((4, 3), -1))
    K, V = (torch.zeros(8 * 2 * 16 * 64 * 2 + 16, dtype=torch.uint8, device="cuda") for _ in range(2))
    before = handle.launch_count()

    def reorder(status, desc=None, beams=2, parents=parents, src=table[:4], dst=table[4:8], copies=copies):
        with pytest.raises(rk.RestKVError) as e:
            handle.paged_reorder(desc or cache(), beams, parents, lengths, src, dst, copies)
        assert e.value.status == status

    reorder(rk.ERR_INVALID_ARG, beams=3)
    reorder(rk.ERR_INVALID_ARG, beams=0)
    reorder(rk.ERR_INVALID_ARG, parents=None)
    reorder(rk.ERR_INVALID_ARG, copies=None)
    reorder(rk.ERR_INVALID_ARG, dst=None)
    reorder(rk.ERR_INVALID_ARG, dst=table[1:5])       # neither the table nor apart from it
    reorder(rk.ERR_INVALID_ARG, desc=cache(page_rows=24))
    reorder(rk.ERR_UNSUPPORTED, desc=cache(lengths_per_head=1))
    reorder(rk.ERR_UNSUPPORTED, desc=cache(batch=130), beams=65)

    def copy(status, desc=None, K=K, V=V, copies=copies, n=4, layers=1, layer_bytes=0):
        with pytest.raises(rk.RestKVError) as e:
            handle.paged_copy(desc or cache(), copies, K, V, n_copies=n, n_layers=layers, layer_bytes=layer_bytes)
        assert e.value.status == status

    copy(rk.ERR_INVALID_ARG, K=None)
    copy(rk.ERR_INVALID_ARG, V=V[8:])
    copy(rk.ERR_INVALID_ARG, n=0)
    copy(rk.ERR_INVALID_ARG, layers=0)
    copy(rk.ERR_INVALID_ARG, layer_bytes=-16)
    copy(rk.ERR_INVALID_ARG, layers=2, layer_bytes=8 * 2 * 16 * 64 * 2 - 16)
    copy(rk.ERR_INVALID_ARG, layer_bytes=8 * 2 * 16 * 64 * 2 + 8)
    copy(rk.ERR_INVALID_ARG, desc=cache(head_dim=0))
    copy(rk.ERR_UNSUPPORTED, n=2 ** 30, layers=2)
    assert handle.launch_count() == before


# ---- a search, whole ------------------------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_a_search_over_pages_is_one_over_copies(handle, fmt):
    """Some steps of a search with the cache in pages that hypotheses share, and with a cache of its own for each that is copied at every step: the same
    rows, attention to the same bits."""
    requests, beams, H, d, R, vocab, prompt, steps = 2, 4, 2, 64, 16, 500, 21, 40
    g = torch.Generator("cuda").manual_seed(11)
    S, width = requests * beams, -(-(prompt + steps) // R) + 1
    embed, head = torch.randn(vocab, 3, H, d, generator=g, device="cuda").to(torch.bfloat16), torch.randn(H * d, vocab, generator=g, device="cuda") * 0.3
    format = dict(page_format=rk.PAGES_BF16) if fmt == "bf16" else dict(page_format=rk.PAGES_INT4, group=32)
    n_pages = requests * width * (beams + 1)
    desc = rk.make_paged(S, H, H, d, page_rows=R, n_pages=n_pages, table_width=width, **format)
    page = handle.paged_page_bytes(desc)
    K, V = (torch.full((n_pages, page), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
    free = list(range(n_pages))
    table = torch.full((S, width), -1, dtype=torch.int32, device="cuda")
    full = prompt // R
    for r in range(requests):
        common = [free.pop() for _ in range(full)]
        for k in range(beams):
            table[r * beams + k] = dev_i32(common + [free.pop()] + [-1] * (width - full - 1))
    # the prompt goes into the first hypothesis of every request
    first = rk.make_paged(requests, H, H, d, page_rows=R, n_pages=n_pages, table_width=width, **format)
    k0, v0 = (torch.randn(requests, H, prompt, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    handle.paged_append(first, prompt, k0, v0, K, V, dev_i32([prompt] * requests), table[::beams].contiguous())
    # the other cache: a sequence of pages of its own for each
    own = rk.make_paged(S, H, H, d, page_rows=R, n_pages=S * width, table_width=width, **format)
    own_table = torch.arange(S * width, dtype=torch.int32, device="cuda").view(S, width)
    own_K, own_V = (torch.full((S * width, page), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
    handle.paged_append(own, prompt, k0.repeat_interleave(beams, 0), v0.repeat_interleave(beams, 0), own_K, own_V, dev_i32([prompt] * S), own_table)

    sel = rk.make_beams(requests, beams, vocab, beams, rk.F32)
    ws, ws_sel = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in (handle.paged_workspace_bytes(desc, 1), handle.beam_workspace_bytes(sel)))
    scores = torch.full((requests, beams), NEG_INF, device="cuda")
    scores[:, 0] = 0
    logits = torch.randn(S, vocab, generator=g, device="cuda")
    parents, tokens = (torch.empty(requests, beams, dtype=torch.int32, device="cuda") for _ in range(2))
    copies, dropped = torch.empty(S, 3, dtype=torch.int32, device="cuda"), torch.empty_like(table)
    copied = returned = 0
    for step in range(steps):
        rows = prompt + step
        handle.beam_select(sel, logits, scores, parents, tokens, scores, ws_sel)
        handle.paged_reorder(desc, beams, parents, dev_i32([rows] * S), table, table, copies, dropped=dropped)
        handle.paged_copy(desc, copies, K, V)
        copied += int((copies[:, 0] >= 0).sum())
        back = dropped[dropped >= 0].tolist()
        returned += len(back)
        free += back
        if rows % R == 0:                        # a page of its own for every hypothesis' next rows
            table[:, rows // R] = dev_i32([free.pop() for _ in range(S)])
        who = (torch.arange(requests, device="cuda")[:, None] * beams + parents).view(-1).long()
        own_K, own_V = (x.view(S, width, page)[who].reshape(S * width, page).contiguous() for x in (own_K, own_V))
        qkv = embed[tokens.view(-1).long()].permute(1, 0, 2, 3).unsqueeze(3).contiguous()      # [3, S, H, 1, d]
        lengths = dev_i32([rows + 1] * S)
        out, own_out = (torch.empty(S, H, 1, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for c, t, k, v, o in ((desc, table, K, V, out), (own, own_table, own_K, own_V, own_out)):
            handle.paged_append(c, 1, qkv[1], qkv[2], k, v, lengths, t)
            handle.paged_attend(c, 1, qkv[0], k, v, lengths, t, o, ws)
        assert torch.equal(out, own_out), step
        logits = (out.float().view(S, H * d) @ head).contiguous()
    assert handle.poll_status() == rk.RESTKV_OK
    assert copied > 0 and returned > 0           # the search has branched, and branches have died
    named = table[table >= 0]
    assert not set(named.tolist()) & set(free)
