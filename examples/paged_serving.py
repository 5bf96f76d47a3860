"""A small multi-LoRA decoder served over a paged cache, all of it through the
framework's entry points: every adapter's prompt is run once and its pages are
shared by the adapter's requests; then the requests' own prompts in one batch;
then decode steps of a token each.

    python examples/paged_serving.py [--layers 2] [--requests 24] [--steps 8]

Weights and inputs are random; a step's input stands in for the embedding of the
token that sampling would give.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_05483_amd import paged, plora  # noqa: E402

BF16 = torch.bfloat16


class Model:
    """Attention layers: q, k, v and output projections, each with a stack of
    adapters; no norms or MLP, so that what the framework does stays in view."""

    def __init__(self, layers=2, h=512, heads=8, kv_heads=2, adapters=4, rank=8, seed=0,
                 device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        mk = lambda *s, std: torch.randn(s, device=device, generator=g).mul_(std).to(BF16)
        self.h, self.heads, self.kv_heads, self.adapters = h, heads, kv_heads, adapters
        self.d, self.device, self.layers = h // heads, device, []
        kv = kv_heads * self.d
        i64 = dict(dtype=torch.int64, device=device)
        ranks = torch.full((adapters,), rank, dtype=torch.int32, device=device)
        scales = torch.full((adapters,), 0.5, device=device)
        for _ in range(layers):
            weights = [mk(h, w, std=h ** -0.5) for w in (h, kv, kv)] + [mk(h, h, std=h ** -0.5)]
            stacks = []
            for w in (h, kv, kv, h):
                A, B = mk(adapters * h * rank, std=h ** -0.5), mk(adapters * rank * w, std=0.2)
                stacks.append(plora.Adapters(A, B, torch.arange(adapters, **i64) * h * rank,
                                             torch.arange(adapters, **i64) * rank * w, ranks,
                                             scales, h, w, rank))
            self.layers.append((weights, stacks))
        self.turns = paged.rope_turns(self.d, device=device)


class Server:
    """The caches of all layers, the block table of the running requests and the
    list of free pages."""

    def __init__(self, model, pages=256, page_size=16, max_pages=32):
        self.m, self.page_size, self.max_pages = model, page_size, max_pages
        self.caches = [paged.KVCache.empty(pages, page_size, model.kv_heads, model.d,
                                           device=model.device) for _ in model.layers]
        i32 = dict(dtype=torch.int32, device=model.device)
        self.free, self.head = torch.arange(pages, **i32), torch.zeros(1, **i32)

    def step(self, x, past, new, table, adapter, prefix_len=None):
        """One batch: x [T, h] are the new tokens' inputs, new (a list) their
        numbers by request, past and adapter int32 [batch].  Returns the outputs
        and the requests' new lengths."""
        m, T, B = self.m, x.shape[0], len(new)
        dev, d = m.device, m.d
        new_dev = torch.tensor(new, dtype=torch.int32, device=dev)
        step = paged.Step(B, T, self.page_size, self.max_pages, device=dev, table=table)
        head = torch.zeros_like(self.head)
        paged.kv_plan(past, new_dev, self.free, self.head, head, step)
        self.head = head
        # the batch's requests by adapter: who shares a prefix ...
        groups = plora.Segments(B, m.adapters, device=dev)
        plora.segment(adapter, groups)
        plan = paged.AttnPlan(step, m.heads, m.kv_heads, d, max_q=max(new),
                              shared=prefix_len is not None, device=dev)
        if prefix_len is not None:
            paged.attn_plan(step, plan, groups, prefix_len)
        else:
            paged.attn_plan(step, plan)
        # ... and its tokens by adapter, for the projections
        idx = adapter.repeat_interleave(new_dev, output_size=T).contiguous()
        segs = plora.Segments(T, m.adapters, device=dev)
        plora.segment(idx, segs)
        ws = plora.Workspace(T, m.layers[0][1][:3], device=dev)
        for (weights, stacks), cache in zip(m.layers, self.caches):
            q, k, v = (x @ w for w in weights[:3])
            plora.apply_multi(x, stacks[:3], segs, [q, k, v], ws)
            q, k, v = q.view(T, m.heads, d), k.view(T, m.kv_heads, d), v.view(T, m.kv_heads, d)
            out = torch.empty_like(q)
            paged.run_layers(step, plan, [(q, k, v, cache, out)], m.turns, d ** -0.5)
            out = out.view(T, m.h)
            y = out @ weights[3]
            plora.apply(out, stacks[3], segs, y, ws)
            x = x + y
        return x, step.kv_len


def serve(model, requests=24, steps=8, prefix=64, prompt=40, share=True, seed=1, pages=1024):
    """Runs it all; returns every step's outputs and the inputs they came from,
    by request: (inputs [n, h], outputs [n, h], adapter)."""
    dev = model.device
    g = torch.Generator(device="cpu").manual_seed(seed)
    mk = lambda n: torch.randn((n, model.h), generator=g).to(BF16).to(dev)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=dev)
    s = Server(model, pages=pages)
    N = model.adapters
    # the adapters' prompts, whole pages each
    assert prefix % s.page_size == 0
    lead = i32([[0] * s.max_pages] * N)
    xp = mk(N * prefix)
    yp, _ = s.step(xp, i32([0] * N), [prefix] * N, lead, i32(list(range(N))))
    own = [[a % N, [xp[a % N * prefix:(a % N + 1) * prefix]],
            [yp[a % N * prefix:(a % N + 1) * prefix]]] for a in range(requests)]
    adapter = i32([a for a, _, _ in own])
    table = lead[adapter.long()].contiguous()
    past = i32([prefix] * requests)
    lens = i32([prefix] * N) if share else None
    for t in range(steps + 1):
        new = [1 + (7 * r) % prompt for r in range(requests)] if t == 0 else [1] * requests
        x = mk(sum(new))
        y, past = s.step(x, past, new, table, adapter, lens)
        at = 0
        for r, n in enumerate(new):
            own[r][1].append(x[at:at + n])
            own[r][2].append(y[at:at + n])
            at += n
    return [(torch.cat(x), torch.cat(y), a) for a, x, y in own]


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--requests", type=int, default=24)
    ap.add_argument("--steps", type=int, default=8)
    args = ap.parse_args()
    model = Model(layers=args.layers)
    serve(model, args.requests, 1)
    for share in (False, True):
        torch.cuda.synchronize()
        t = time.perf_counter()
        out = serve(model, args.requests, args.steps, share=share)
        torch.cuda.synchronize()
        t = time.perf_counter() - t
        n = sum(y.shape[0] for _, y, _ in out)
        print(f"shared prefixes {share}: {n} tokens of {args.requests} requests in {t * 1e3:.1f} ms")


if __name__ == "__main__":
    main()
