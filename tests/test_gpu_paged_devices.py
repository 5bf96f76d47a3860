"""One host tensor among a call's GPU tensors is refused before anything is launched:
its address would be no address to a kernel."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_paged import G, P  # noqa: E402, F401

I32, I64, BF = torch.int32, torch.int64, torch.bfloat16


def refused(call, args):
    """Runs with all on the GPU, then with each argument on the host in turn."""
    call(**args)
    torch.cuda.synchronize()
    for name, t in args.items():
        with pytest.raises(ValueError, match="device"):
            call(**dict(args, **{name: t.cpu()}))


def test_each_argument(G, P):
    z = lambda *s, dt=BF: torch.zeros(s, dtype=dt, device="cuda")
    i = lambda n, dt=I32: torch.zeros(n, dtype=dt, device="cuda")
    step = G.Step(2, 5, 16, 4)
    refused(lambda **a: G.kv_plan(a["past"], a["new"], a["free"], a["head"], a["next"], step),
            dict(past=i(2), new=i(2), free=i(3), head=i(1), next=i(1)))
    refused(lambda **a: G.rope(a["x"], a["pos"], a["turns"], a["out"]),
            dict(pos=i(5), turns=i(32, I64), x=z(5, 4, 64), out=z(5, 4, 64)))
    cache = G.KVCache(z(3, 2, 16, 64), z(3, 2, 16, 64))
    refused(lambda **a: G.rope_append(a["q"], a["k"], a["v"], a["pos"], a["slot"], a["turns"],
                                      cache, a["out"]),
            dict(q=z(5, 4, 64), k=z(5, 2, 64), v=z(5, 2, 64), pos=i(5), slot=i(5, I64),
                 turns=i(32, I64), out=z(5, 4, 64)))
    plan = G.AttnPlan(step, 4, 2, 64, max_q=3, shared=True)
    segs = P.Segments(2, 1)
    P.segment(i(2), segs)
    refused(lambda **a: G.attn_plan(step, plan, segs, a["prefix"]), dict(prefix=i(1)))
    refused(lambda **a: G.attn_paged(a["q"], cache, step, plan, 0.1, a["out"]),
            dict(q=z(5, 4, 64), out=z(5, 4, 64)))
    # and what the calls are given beside tensors
    q = z(5, 4, 64)
    host = G.Step(2, 5, 16, 4, device="cpu")
    cold = G.KVCache(cache.k.cpu(), cache.v.cpu())
    for call in (lambda: G.kv_plan(i(2), i(2), i(3), i(1), i(1), host),
                 lambda: G.attn_plan(host, plan),
                 lambda: G.attn_plan(step, plan, P.Segments(2, 1, device="cpu"), i(1)),
                 lambda: G.attn_plan(step, G.AttnPlan(step, 4, 2, 64, max_q=3, device="cpu")),
                 lambda: G.attn_paged(q, cache, host, plan, 0.1, q.clone()),
                 lambda: G.attn_paged(q, cold, step, plan, 0.1, q.clone()),
                 lambda: G.KVCache(cache.k, cache.v.cpu()),
                 lambda: G.Step(2, 5, 16, 4, table=torch.zeros((2, 4), dtype=I32))):
        with pytest.raises(ValueError, match="device"):
            call()
