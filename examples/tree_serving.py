"""Serving with trees of drafted tokens, all of it through the framework's entry points:
each request's next tokens are guessed from what followed the same token before (several
guesses make a tree), one step of the model looks at all of them, the longest path that
it agrees with is kept, its keys are moved together and the pages behind are given back.
Halfway every request is continued by two, the second with another token, which share
their pages; at the end all have ended and every page is free again.

    python examples/tree_serving.py [--requests 8] [--steps 24]

Weights are random (the multi-LoRA decoder of paged_serving.py, with an embedding whose
transpose gives the logits).
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from paged_serving import BF16, Model  # noqa: E402

from paper_2608_05483_amd import pages, paged, plora, tree  # noqa: E402


def draft(history, root, nodes, width):
    """A tree of up to ``nodes`` tokens below root: up to ``width`` of the tokens that
    followed each node's token in the request's history, the latest first, level by
    level.  Returns tokens and parents."""
    followers = {}
    for a, b in zip(history, history[1:]):
        seen = followers.setdefault(a, [])
        if b in seen:
            seen.remove(b)
        seen.insert(0, b)
    tokens, parents, at = [root], [-1], 0
    while at < len(tokens) and len(tokens) < nodes:
        for b in followers.get(tokens[at], [])[:width]:
            if len(tokens) < nodes:
                tokens.append(b)
                parents.append(at)
        at += 1
    return tokens, parents


class Server:
    """The caches of all layers, who holds their pages, and the running requests."""

    def __init__(self, model, vocab=64, n_pages=1024, page_size=16, max_pages=64, seed=3):
        self.m, self.page_size, self.max_pages = model, page_size, max_pages
        dev = model.device
        g = torch.Generator(device=dev).manual_seed(seed)
        self.embed = torch.randn((vocab, model.h), device=dev, generator=g).to(BF16)
        self.layers = [paged.KVCache.empty(n_pages, page_size, model.kv_heads, model.d, device=dev)
                       for _ in model.layers]
        self.caches = pages.Caches(self.layers)
        self.pool = pages.PagePool.empty(n_pages, device=dev)
        self.head = self.i32([0])
        self.table = torch.zeros((0, max_pages), dtype=torch.int32, device=dev)
        self.kv_len = self.i32([])

    def i32(self, a):
        return torch.tensor(a, dtype=torch.int32, device=self.m.device)

    def remap(self, table, kv_len, src, keep=None):
        """The running requests become those of src, each with its first keys."""
        out = pages.Remap(len(kv_len), len(src), self.page_size, self.max_pages,
                          device=self.m.device)
        head = torch.zeros_like(self.head)
        pages.kv_remap(table, kv_len, self.i32(src), keep, self.pool, self.head, head, out)
        pages.kv_copy(self.caches, out)
        self.table, self.kv_len, self.head = out.table, out.kv_len, head

    def step(self, tokens, parents, given, adapter):
        """One step over every request's nodes (lists by request).  Returns the outputs
        of all nodes, the accepted paths and the next tokens."""
        m, d, dev = self.m, self.m.d, self.m.device
        new = [len(t) for t in tokens]
        B, T = len(new), sum(new)
        flat = torch.tensor(sum(tokens, []), dtype=torch.int64, device=dev)
        parent, new_dev = self.i32(sum(parents, [])), self.i32(new)
        step = paged.Step(B, T, self.page_size, self.max_pages, device=dev, table=self.table)
        head = torch.zeros_like(self.head)
        paged.kv_plan(self.kv_len, new_dev, self.pool.free_pages, self.head, head, step)
        self.head = head
        t = tree.Tree(step, device=dev)
        tree.tree_plan(parent, step, t)
        plan = paged.AttnPlan(step, m.heads, m.kv_heads, d, max_q=max(new), device=dev)
        paged.attn_plan(step, plan)
        idx = adapter.repeat_interleave(new_dev, output_size=T).contiguous()
        segs = plora.Segments(T, m.adapters, device=dev)
        plora.segment(idx, segs)
        ws = plora.Workspace(T, m.layers[0][1][:3], device=dev)
        x = self.embed[flat]
        for (weights, stacks), cache in zip(m.layers, self.layers):
            q, k, v = (x @ w for w in weights[:3])
            plora.apply_multi(x, stacks[:3], segs, [q, k, v], ws)
            q, k, v = q.view(T, m.heads, d), k.view(T, m.kv_heads, d), v.view(T, m.kv_heads, d)
            out = torch.empty_like(q)
            tree.run_layers(step, plan, t, [(q, k, v, cache, out)], m.turns, d ** -0.5)
            out = out.view(T, m.h)
            y = out @ weights[3]
            plora.apply(out, stacks[3], segs, y, ws)
            x = x + y
        target = (x @ self.embed.t()).argmax(-1)
        a = tree.Accepted(step, dtype=torch.int64, device=dev)
        tree.tree_accept(parent, flat, target, step, a, given=self.i32(given))
        pages.kv_compact(self.caches, step, a.path, a.count)
        self.remap(step.table, step.kv_len, list(range(B)), keep=a.kv_len)
        count, path, at, paths = a.count.tolist(), a.path.tolist(), 0, []
        for n, c in zip(new, count):
            paths.append(path[at:at + c])
            at += n
        return x, paths, a.token.tolist()


def serve(model, requests=8, steps=24, nodes=12, width=2, prompt=20, vocab=64, seed=1,
          n_pages=1024):
    """Runs it; returns by request (tokens with the model's output for each, adapter,
    tokens kept a step) and the server."""
    s = Server(model, vocab=vocab, n_pages=n_pages)
    g = torch.Generator().manual_seed(seed)
    run = [dict(tokens=torch.randint(0, vocab, (1 + (7 * r) % prompt,), generator=g).tolist(),
                adapter=r % model.adapters, outputs=[], kept=[]) for r in range(requests)]
    s.remap(s.table, s.kv_len, [-1] * requests)
    for i in range(steps):
        if i == steps // 2:
            # every request is continued by two, the second with another token
            s.remap(s.table, s.kv_len, [r for r in range(len(run)) for _ in range(2)])
            run = [dict(x, tokens=list(x["tokens"]), outputs=list(x["outputs"]),
                        kept=list(x["kept"])) for x in run for _ in range(2)]
            for x in run[1::2]:
                x["tokens"][-1] = (x["tokens"][-1] + 1) % vocab
        drafts = []
        for x in run:
            if i == 0:
                n = len(x["tokens"])
                drafts.append((list(x["tokens"]), [j - 1 for j in range(n)]))
            else:
                drafts.append(draft(x["tokens"], x["tokens"][-1], nodes, width))
        given = [len(x["tokens"]) if i == 0 else 1 for x in run]
        y, paths, token = s.step([t for t, _ in drafts], [p for _, p in drafts], given,
                                 s.i32([x["adapter"] for x in run]))
        at = 0
        for x, (t, _), path, nxt in zip(run, drafts, paths, token):
            x["outputs"] += [y[at + j] for j in path]
            # (the first node is the last token already there)
            x["tokens"] += [t[j] for j in path[1:]] if i else []
            x["tokens"].append(nxt)
            x["kept"].append(len(path))
            at += len(t)
    s.remap(s.table, s.kv_len, [])
    return run, s


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--steps", type=int, default=24)
    args = ap.parse_args()
    model = Model(layers=2)
    serve(model, args.requests, 2)
    for width, nodes in ((1, 1), (2, 12)):
        torch.cuda.synchronize()
        t = time.perf_counter()
        run, _ = serve(model, args.requests, args.steps, nodes=nodes, width=width)
        torch.cuda.synchronize()
        t = time.perf_counter() - t
        kept = [n for x in run for n in x["kept"][1:]]
        print(f"trees of up to {nodes}: {sum(kept) / len(kept):.2f} tokens a request and step, "
              f"{t / args.steps * 1e3:.2f} ms a step")


if __name__ == "__main__":
    main()
