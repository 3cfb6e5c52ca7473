"""A population decoding: the projections of every candidate, and between them the 4-bit key/value cache.

K candidates share quantised base weights and differ in the singular values of their LoRA factors, so a prompt's keys and
values are a candidate's own.  Each candidate reads the same prompt into the cache once; its samples are forked from there
(whole pages shared, the partly filled last one copied) and decode together, one recorded step a token.  In the middle some
samples end: their pages go back and the pages in use are moved together.  Weights are random and a step's output,
normalised, is the next step's input: what is shown is the order of the calls, not language.

    python examples/population_decode.py [--candidates 4] [--samples 4] [--layers 2] [--prompt 200] [--steps 48]
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import essa_workloads as wl  # noqa: E402
import paper_2507_04453_amd as essa  # noqa: E402


class Model:
    """The q, k, v and o projections of a few layers, and every candidate's singular values."""

    def __init__(self, ctx, layers, hidden, kv, rank, head_dim, candidates):
        self.ctx, self.layers, self.hidden, self.head_dim = ctx, layers, hidden, head_dim
        self.q_heads, self.kv_heads = hidden // head_dim, kv // head_dim
        self.projs, self.sigma = [], []
        for l in range(layers):
            projs, sigmas = [], []
            for p, w in enumerate(wl.make_layer(hidden, kv, rank, "int8", layer=l)):
                proj = essa.Projection(ctx, w.Wq, w.scales, None, w.A, w.B, essa.QUANT_INT8_PERCH)
                dA, dB = wl.sigma_perturbation(candidates, 1, rank, 0.05, 4 * l + p)
                sA, sB = proj.spectrum()
                projs.append(proj)
                sigmas.append(tuple(torch.from_numpy(s + d[:, 0]).float().cuda().contiguous() for s, d in ((sA, dA), (sB, dB))))
            self.projs.append(projs)
            self.sigma.append(sigmas)

    def buffers(self, rows):
        """Activations of a call of so many rows, with everything that a step computes on the way: a recorded step writes where it wrote
        when it was recorded, so nothing of it may be memory that somebody else is given later."""
        new = lambda width, dtype=torch.bfloat16: torch.empty(rows, width, device="cuda", dtype=dtype)
        return {"x": new(self.hidden), "h": new(self.hidden), "q": new(self.hidden), "k": new(self.kv_heads * self.head_dim),
                "v": new(self.kv_heads * self.head_dim), "a": new(self.hidden), "o": new(self.hidden),
                "x32": new(self.hidden, torch.float32), "square": new(self.hidden, torch.float32), "norm": new(1, torch.float32)}

    def groups(self, buf, row2cand):
        """The marshalled projections of every layer: q, k and v together, then o."""
        out = []
        for projs, sigmas in zip(self.projs, self.sigma):
            item = lambda p, x, y: (projs[p], buf[x], row2cand, *sigmas[p], buf[y])
            out.append((essa.ForwardGroup([item(0, "h", "q"), item(1, "h", "k"), item(2, "h", "v")]), essa.ForwardGroup([item(3, "a", "o")])))
        return out

    def forward(self, kv, buf, groups, batch):
        """x <- x + o(attention(q, cache with k and v)) for every layer; the cache has room for the rows already.  Allocates nothing."""
        x32, norm = buf["x32"], buf["norm"]
        for l, (qkv, o) in enumerate(groups):
            x32.copy_(buf["x"])
            torch.mean(torch.mul(x32, x32, out=buf["square"]), 1, keepdim=True, out=norm)
            norm.add_(1e-6).rsqrt_()
            buf["h"].copy_(x32.mul_(norm))
            essa.essa_svdlora_forward_group(self.ctx, qkv)
            essa.essa_kv_append(self.ctx, kv, l, buf["k"], buf["v"], batch)
            essa.essa_kv_attention(self.ctx, kv, l, buf["q"], buf["a"], batch, scale=0.02 / math.sqrt(self.head_dim))
            essa.essa_svdlora_forward_group(self.ctx, o)
            buf["x"] += buf["o"].mul_(0.05)


def run(candidates=4, samples=4, layers=2, hidden=3584, kv_width=512, rank=16, head_dim=128, prompt=200, steps=48, record=True, quiet=False):
    """Returns the last step's activations, the cache's lengths and the number of pages in use."""
    say = (lambda *a: None) if quiet else (lambda *a: print(*a, flush=True))
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = essa.Context(0, stream)
        model = Model(ctx, layers, hidden, kv_width, rank, head_dim, candidates)
        K, n = candidates, candidates * samples
        i32 = lambda x: torch.tensor(list(x), dtype=torch.int32, device="cuda")
        pages = K * -(-prompt // 64) + n * (-(-(steps + 64) // 64) + 1)
        kv = essa.KvCache(ctx, layers, model.kv_heads, head_dim, pages, page_tokens=64, max_seqs=K + n, max_tokens=prompt + steps)

        # prompts: sequence c is candidate c's, all rows of one candidate next to one another
        g = torch.Generator(device="cuda")
        g.manual_seed(1)
        tokens = torch.randn(prompt, hidden, generator=g, device="cuda")
        buf = model.buffers(K * prompt)
        buf["x"].copy_(tokens.repeat(K, 1))
        seqs, served = i32(range(K)), torch.empty(K, dtype=torch.int32, device="cuda")
        essa.essa_kv_extend(ctx, kv, seqs, i32([prompt] * K), served)
        model.forward(kv, buf, model.groups(buf, i32(c for c in range(K) for _ in range(prompt))),
                      essa.KvBatch(served, i32(prompt * c for c in range(K + 1)), K * prompt))
        last = buf["x"].view(K, prompt, hidden)[:, -1]

        # samples: sequences K .. K + n - 1, forked off their candidate's prompt, which is then let go
        mine = i32(K + i for i in range(n))
        essa.essa_kv_fork(ctx, kv, i32(i // samples for i in range(n)), mine, served=torch.empty_like(mine))
        essa.essa_kv_free(ctx, kv, seqs)
        torch.cuda.synchronize()
        say("%d candidates, %d prompt rows each; %d samples share their pages: %d of %d pages in use" %
            (K, prompt, n, int((kv.refs > 0).sum()), kv.n_pages))

        buf = model.buffers(n)
        buf["x"].copy_(last.repeat_interleave(samples, 0))
        groups = model.groups(buf, i32(i // samples for i in range(n)))
        one, alive, served = i32([1] * n), mine.clone(), torch.empty_like(mine)
        batch = essa.KvBatch(served)               # a sample that has ended, or found no page, is skipped from here on

        def step():
            essa.essa_kv_extend(ctx, kv, alive, one, served)
            model.forward(kv, buf, groups, batch)

        step()                                     # unrecorded: scratch grows to its size
        graph = None
        if record:
            torch.cuda.synchronize()
            ctx.graph_begin()
            step()
            graph = ctx.graph_end()
        replay = graph.launch if record else step
        used = torch.empty(1, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        for t in range(1, steps):
            if t == steps // 2:
                ended = mine[::3].contiguous()
                alive[::3] = -1
                essa.essa_kv_free(ctx, kv, ended)
                essa.essa_kv_compact(ctx, kv, used_out=used)
            replay()
        torch.cuda.synchronize()
        dt = time.perf_counter() - t0
        say("%d steps of %d samples in %.1f ms (%.0f us a step of %d layers); %d pages in use, all below %d" %
            (steps - 1, n, dt * 1e3, dt * 1e6 / (steps - 1), layers, int((kv.refs > 0).sum()), int(torch.nonzero(kv.refs).max()) + 1))
        out = buf["x"].clone(), kv.len.clone(), int((kv.refs > 0).sum())
        assert torch.isfinite(out[0]).all()
        if graph is not None:
            graph.close()
        kv.close()
        ctx.close()
    return out


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    for name, default in (("candidates", 4), ("samples", 4), ("layers", 2), ("prompt", 200), ("steps", 48)):
        ap.add_argument("--" + name, type=int, default=default)
    run(**vars(ap.parse_args()))
