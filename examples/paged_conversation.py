"""One attention layer of a conversation over a paged 4-bit cache, with eviction between the turns.

    python examples/paged_conversation.py [--prompt 4096] [--budget 1024] [--generate 48] [--turn 256]

The prompt's rows are rotated and appended to the pages, and its tokens attend to them (restkv_paged_append, restkv_paged_attend); the
rows are read back (restkv_paged_read), scored and evicted (restkv_evict), and what is kept becomes the cache's rows again.  Then tokens
are generated one at a time, a second turn comes as a chunk, and the cache, grown by both, is evicted again.  Everything is enqueued on
one stream; the host waits at the end only.
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2605_08840_b200 import binding as rk  # noqa: E402


class PagedLayer:
    """The pages of one layer, what lies in them, and the calls that a model's attention makes."""

    def __init__(self, handle, batch, heads, kv_heads, dim, most_rows, most_tokens, page_rows=64, group=64, positions=1 << 16):
        self.h, self.batch, self.heads, self.kv_heads, self.dim = handle, batch, heads, kv_heads, dim
        width = -(-most_rows // page_rows)
        self.cache = rk.make_paged(batch, heads, kv_heads, dim, rk.PAGES_INT4, page_rows, batch * width, width, group)
        page = handle.paged_page_bytes(self.cache)
        self.K, self.V = (torch.empty(batch * width, page, dtype=torch.uint8, device="cuda") for _ in range(2))
        # any pages will do; a server hands them out as sequences grow and takes them back after an eviction
        self.table = torch.randperm(batch * width, device="cuda").to(torch.int32).view(batch, width)
        self.rows = 0
        angles = torch.arange(positions, device="cuda")[:, None] * 500000.0 ** (-torch.arange(0, dim, 2, device="cuda") / dim)
        self.rotation = rk.make_rotation(angles.cos().float().contiguous(), angles.sin().float().contiguous(), dim)
        self.workspace = torch.empty(max(handle.paged_workspace_bytes(self.cache, t) for t in (1, most_tokens)), dtype=torch.uint8, device="cuda")

    def lengths(self):
        return torch.full((self.batch,), self.rows, dtype=torch.int32, device="cuda")

    def step(self, Q, K, V, position):
        """Tokens [batch, heads, t, dim] whose first is at `position`: (their rotated queries, their attention over all rows so far)."""
        t = K.shape[2]
        self.rows += t
        lengths = self.lengths()
        positions = torch.arange(position, position + t, dtype=torch.int32, device="cuda").repeat(self.batch, 1)
        turned, out = (torch.empty(self.batch, self.heads, t, self.dim, dtype=Q.dtype, device="cuda") for _ in range(2))
        self.h.paged_append(self.cache, t, K, V, self.K, self.V, lengths, self.table, positions=positions, rotation=self.rotation, Q=Q, Q_out=turned)
        self.h.paged_attend(self.cache, t, turned, self.K, self.V, lengths, self.table, out, self.workspace)
        return turned, out

    def read(self):
        K, V = (torch.empty(self.batch, self.kv_heads, self.rows, self.dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.h.paged_read(self.cache, self.K, self.V, self.lengths(), self.table, self.rows, K, V)
        return K, V

    def evict(self, observed, budget):
        """Keeps `budget` rows of every head by the last queries, [batch, heads, w, dim], the rows of those tokens among them."""
        K, V = self.read()
        w = observed.shape[2]
        shape = rk.make_shape(self.batch, self.heads, self.kv_heads, self.dim, self.rows, w, causal_tail=w)
        indices = torch.empty(self.batch, self.kv_heads, budget, dtype=torch.int32, device="cuda")
        kept_K, kept_V = (torch.empty(self.batch, self.kv_heads, budget, self.dim, dtype=K.dtype, device="cuda") for _ in range(2))
        workspace = torch.empty(self.h.workspace_bytes(shape, budget), dtype=torch.uint8, device="cuda")
        self.h.evict(shape, observed.contiguous(), K, V, 0.9, rk.fixed_pool(7), budget, indices, kept_K, kept_V, workspace)
        self.rows = budget                         # rotated already: they go back as they are
        self.h.paged_append(self.cache, budget, kept_K, kept_V, self.K, self.V, self.lengths(), self.table)
        return indices


def run(prompt=4096, budget=1024, generate=48, turn=256, window=32, batch=2, heads=32, kv_heads=8, dim=128, seed=0):
    """The last generated token's rotated query and attention, with the rows that it was over; rows of the cache after each stage."""
    handle = rk.Handle()
    g = torch.Generator(device="cuda").manual_seed(seed)

    def project(t):                                # stands for a model's projections: [batch, t, heads, dim], read as [batch, heads, t, dim]
        x = torch.randn(batch, t, heads + 2 * kv_heads, dim, generator=g, device="cuda").to(torch.bfloat16).transpose(1, 2)
        return x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]

    layer = PagedLayer(handle, batch, heads, kv_heads, dim, max(prompt, budget + generate + turn) + 2, max(prompt, turn))
    position, rows = prompt, [prompt]
    turned, _ = layer.step(*project(prompt), 0)
    layer.evict(turned[:, :, -window:], budget)
    rows.append(layer.rows)
    for _ in range(generate):
        layer.step(*project(1), position)
        position += 1
    rows.append(layer.rows)
    turned, _ = layer.step(*project(turn), position)
    position += turn
    rows.append(layer.rows)
    layer.evict(turned[:, :, -window:], budget)
    rows.append(layer.rows)
    turned, out = layer.step(*project(1), position)
    K, V = layer.read()
    if handle.poll_status() != rk.RESTKV_OK:
        raise RuntimeError("a row, page or position was out of range")
    launches = handle.launch_count()
    handle.close()
    return {"q": turned, "out": out, "K": K, "V": V, "rows": rows, "launches": launches}


def reference(q, K, V):
    """Attention of single tokens over dense rows in 64 bits."""
    b, hq, t, d = q.shape
    group = hq // K.shape[1]
    K, V = (x.double().repeat_interleave(group, 1) for x in (K, V))
    return torch.softmax(q.double() @ K.transpose(2, 3) / d ** 0.5, -1) @ V


def main():
    p = argparse.ArgumentParser()
    for name, value in (("prompt", 4096), ("budget", 1024), ("generate", 48), ("turn", 256)):
        p.add_argument("--" + name, type=int, default=value)
    r = run(**vars(p.parse_args()))
    err = (r["out"].double() - reference(r["q"], r["K"], r["V"])).abs().max()
    print("rows after prompt, eviction, generation, turn, eviction: %s; %d launches" % (r["rows"], r["launches"]))
    print("last token's attention: largest difference from 64 bits %.2e of %.2e" % (float(err), float(r["out"].abs().max())))


if __name__ == "__main__":
    main()
