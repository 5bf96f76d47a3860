"""examples/paged_serving.py: the adapters' projections, the step's plan, rotary
positions, the paged cache and the attention over it, together, against a plain
dense run of every request by itself."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "paged_serving.py")


@pytest.fixture(scope="module")
def E():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    spec = importlib.util.spec_from_file_location("paged_serving", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def dense(model, x, adapter):
    """One request in float64: its whole sequence at once."""
    f = lambda t: t.double()
    n, d, H, KH = x.shape[0], model.d, model.heads, model.kv_heads
    ang = torch.arange(n, dtype=torch.float64, device=x.device)[:, None] * 10000.0 ** (
        -torch.arange(0, d, 2, dtype=torch.float64, device=x.device) / d)
    c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]

    def turn(t):
        a, b = t[..., :d // 2], t[..., d // 2:]
        return torch.cat([a * c - b * s, a * s + b * c], -1)

    def project(y, w, st):
        r = int(st.ranks[adapter])
        A = f(st.A[adapter * st.h_in * r:(adapter + 1) * st.h_in * r]).view(st.h_in, r)
        B = f(st.B[adapter * r * st.h_out:(adapter + 1) * r * st.h_out]).view(r, st.h_out)
        return y @ f(w) + 0.5 * (y @ A) @ B

    x = f(x)
    ahead = torch.ones((n, n), dtype=torch.bool, device=x.device).triu(1)
    for weights, stacks in model.layers:
        q, k, v = (project(x, w, st) for w, st in zip(weights[:3], stacks[:3]))
        q, k, v = turn(q.view(n, H, d)), turn(k.view(n, KH, d)), v.view(n, KH, d)
        out = torch.empty_like(q)
        for h in range(H):
            w = (q[:, h] @ k[:, h * KH // H].t()) * d ** -0.5
            w = torch.softmax(w.masked_fill(ahead, -torch.inf), -1)
            out[:, h] = w @ v[:, h * KH // H]
        x = x + project(out.reshape(n, -1), weights[3], stacks[3])
    return x


@pytest.mark.parametrize("share", [False, True])
def test_serving_matches_a_dense_run(E, share):
    model = E.Model(layers=2)
    for x, y, adapter in E.serve(model, requests=10, steps=4, share=share)[:6]:
        ref = dense(model, x, adapter)
        # each layer rounds to bf16 about ten times on the way (q, k, v, their adapters'
        # sums, the turns, the weights, the output, its projection, the residual):
        # sqrt(2 x 10) roundings of 2^-9 rms, with room of three
        err = (y.double() - ref).norm() / ref.norm()
        assert err <= 3 * 20 ** 0.5 * 2.0 ** -9, float(err)
