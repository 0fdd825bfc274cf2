"""A serving loop over the 8-bit key/value cache: the prompts of a small attention
stack enter the cache in chunks (skm_kv_write, skm_kv_attend on many rows), tokens
are then generated one at a time with the whole step in one CUDA graph
(skm_kv_write of a token, skm_kv_attend on one row), and at the end a sequence's
keys are read back (skm_kv_read) and clustered into an index of the context
(skm_fit).  Weights and prompts are random; the last step's states are
compared with attention over unquantised keys and values in fp32.

    python examples/kv_serve.py --batch 4 --prompt 1000 --chunk 256 --steps 64
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_14648_gb300 as skm  # noqa: E402


class Layer:
    """Random weights of one attention layer, and its cache."""

    def __init__(self, g, width, heads_q, heads, d, page, pages):
        rand = lambda *s: (torch.randn(*s, generator=g, device="cuda") * s[0] ** -0.5).to(torch.bfloat16)  # noqa: E731
        self.heads_q, self.heads, self.d = heads_q, heads, d
        self.w_in, self.w_out = rand(width, (heads_q + 2 * heads) * d), rand(heads_q * d, width)
        self.cache = skm.KVCache(heads, d, page, pages=pages)

    def project(self, x):
        """Rows of (query, key, value) heads: views into one tensor."""
        norm = torch.nn.functional.normalize(x.float(), dim=-1) * x.shape[-1] ** 0.5
        rows = (norm.to(torch.bfloat16) @ self.w_in).view(x.shape[0], -1, self.d)
        return rows.split([self.heads_q, self.heads, self.heads], dim=1)


class Server:
    def __init__(self, batch, most, layers=2, width=256, heads_q=8, heads=2, d=64, page=32, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.batch, self.most = batch, most
        cols = -(-most // page)
        # pages in any order: a sequence finds its own through the table
        order = torch.randperm(batch * cols, generator=g, device="cuda")
        self.table = order.to(torch.int32).view(batch, cols)
        self.layers = [Layer(g, width, heads_q, heads, d, page, batch * cols) for _ in range(layers)]
        self.start = torch.zeros(batch, dtype=torch.int32, device="cuda")
        # one workspace for every call: chunks and single tokens, short contexts and long ones
        self.ws = skm.kv_workspace(self.layers[0].cache, batch, heads_q, batch * most, most, most)

    def forward(self, x, cu, length, max_tokens, max_len):
        """The stack on new rows x; their keys and values enter the caches."""
        for lay in self.layers:
            q, k, v = lay.project(x)
            skm.skm_kv_write(lay.cache, self.table, self.start, cu, k, v, max_tokens)
            out, _ = skm.skm_kv_attend(lay.cache, self.table, length, cu, q, max_tokens, max_len, ws=self.ws)
            x = x + out.view(x.shape[0], -1) @ lay.w_out
        return x

    def prompts(self, xs, chunk):
        """Prompts xs (a list of [n, width]) in chunks; the states of their last tokens."""
        done, last = [0] * len(xs), [None] * len(xs)
        while any(p < len(x) for p, x in zip(done, xs)):
            n = [min(chunk, len(x) - p) for p, x in zip(done, xs)]  # a sequence that is through has no rows
            rows = torch.cat([x[p:p + m] for x, p, m in zip(xs, done, n)])
            cu = torch.tensor([0] + n).cumsum(0).to(torch.int32).cuda()
            length = self.start + cu.diff()
            done = [p + m for p, m in zip(done, n)]
            y = self.forward(rows, cu, length, max(n), max(done))
            self.start.copy_(length)
            for b, m in enumerate(n):
                if m:
                    last[b] = y[int(cu[b + 1]) - 1]
        return torch.stack(last)

    def capture(self):
        """One generated token a sequence as a graph: reads `state`, leaves the next one there."""
        self.cu1 = torch.arange(self.batch + 1, dtype=torch.int32, device="cuda")
        self.state = torch.zeros(self.batch, self.layers[0].w_out.shape[1], dtype=torch.bfloat16, device="cuda")

        def step():
            length = self.start + 1
            y = self.forward(self.state, self.cu1, length, 1, self.most)
            self.state.copy_(y)
            self.start.copy_(length)

        # warm up with all pages absent: a token written here could raise the scale of the block that holds a
        # prompt's last tokens, and their codes would be rounded once more
        at, pages = self.start.clone(), self.table.clone()
        self.table.fill_(-1)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        self.start.copy_(at)
        self.table.copy_(pages)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            step()

    def index(self, b, k, layer=-1, iters=5):
        """Sequence b's keys of one layer, [heads], as k centroids and each token's: points like any others."""
        cache = self.layers[layer].cache
        n = int(self.start[b])
        zero, cu = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda")
        keys = torch.empty(n, cache.heads, cache.d, device="cuda")
        skm.skm_kv_read(cache, self.table[b:b + 1], zero, cu, n, n, skm.DTYPE_F32, out=(keys, None))
        fits = []
        for h in range(cache.heads):
            pts = skm.Points(skm.REPR_F32, keys[:, h].contiguous(), cache.d)
            C, assign, _, obj, _ = skm.skm_fit(pts, k, iters, seed=h)
            fits.append((C, assign, obj[-1]))
        return keys, fits


def full_precision(server, xs, steps):
    """The same run without a cache and in fp32 attention: every sequence's state after `steps` tokens."""
    states = []
    for x in xs:
        past = [[[], []] for _ in server.layers]
        rows = x
        for _ in range(steps + 1):
            y = rows
            for lay, (ks, vs) in zip(server.layers, past):
                q, k, v = lay.project(y)
                ks.append(k.float())
                vs.append(v.float())
                K, V = (torch.cat(t).repeat_interleave(lay.heads_q // lay.heads, 1).transpose(0, 1) for t in (ks, vs))
                s = q.float().transpose(0, 1) @ K.transpose(1, 2) * lay.d ** -0.5
                n, m = s.shape[1:]
                s += torch.full((n, m), -float("inf"), device="cuda").triu(m - n + 1)
                o = (s.softmax(-1) @ V).transpose(0, 1).to(torch.bfloat16)
                y = y + o.reshape(n, -1) @ lay.w_out
            rows = y[-1:]
        states.append(rows[0])
    return torch.stack(states)


def run(batch=4, prompt=1000, chunk=256, steps=64, seed=0):
    server = Server(batch, prompt + steps + 1, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    lengths = [max(1, prompt * (b + 1) // batch) for b in range(batch)]
    xs = [torch.randn(n, 256, generator=g, device="cuda").to(torch.bfloat16) for n in lengths]
    state = server.prompts(xs, chunk)
    server.capture()
    server.state.copy_(state)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(steps):
        server.graph.replay()
    torch.cuda.synchronize()
    step_us = (time.perf_counter() - t) / max(steps, 1) * 1e6
    keys, fits = server.index(batch - 1, min(16, lengths[-1]))
    want = full_precision(server, xs, steps).float()
    error = float((server.state.float() - want).norm() / want.norm())
    return dict(step_us=step_us, error=error, length=server.start.tolist(), keys=keys, fits=fits)


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--batch", type=int, default=4)
    p.add_argument("--prompt", type=int, default=1000)
    p.add_argument("--chunk", type=int, default=256)
    p.add_argument("--steps", type=int, default=64)
    a = p.parse_args()
    r = run(a.batch, a.prompt, a.chunk, a.steps)
    print(f"{a.steps} tokens for {a.batch} sequences of {r['length']} tokens: {r['step_us']:.1f} us a step; "
          f"states within {r['error']:.2e} of attention over unquantised keys and values")
    for h, (C, assign, wcss) in enumerate(r["fits"]):
        print(f"head {h}: {len(C)} centroids of {len(assign)} keys, WCSS {wcss:.4g} of "
              f"{float(((r['keys'][:, h] - r['keys'][:, h].mean(0)) ** 2).sum()):.4g} around the mean")


if __name__ == "__main__":
    main()
