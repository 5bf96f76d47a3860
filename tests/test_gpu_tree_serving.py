"""examples/tree_serving.py: drafted trees, acceptance, moved keys, continued, cut and
ended requests together with the adapters' projections, against a plain dense run of
every request's kept tokens by itself; and what is left of the pool."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_paged_serving import dense  # noqa: E402

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "tree_serving.py")


@pytest.fixture(scope="module")
def E():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    spec = importlib.util.spec_from_file_location("tree_serving", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_drafts(E):
    assert E.draft([1, 2, 3, 1, 4], 1, 6, 2) == ([1, 4, 2, 3, 1, 4], [-1, 0, 0, 2, 3, 4])
    assert E.draft([5], 5, 9, 3) == ([5], [-1])
    assert E.draft([1, 1], 1, 3, 1) == ([1, 1, 1], [-1, 0, 1])


@pytest.mark.parametrize("nodes,width", [(1, 1), (12, 2), (40, 3)])
def test_kept_tokens_match_a_dense_run(E, nodes, width):
    model = E.Model(layers=2)
    run, s = E.serve(model, requests=6, steps=14, nodes=nodes, width=width, vocab=32)
    assert len(run) == 12
    for x in run:
        n = len(x["outputs"])
        assert n == len(x["tokens"]) - 1 == sum(x["kept"])
        y = torch.stack(x["outputs"])
        ref = dense(model, s.embed[torch.tensor(x["tokens"][:n], device=y.device)], x["adapter"])
        # each layer rounds to bf16 about ten times on the way (q, k, v, their adapters'
        # sums, the turns, the weights, the output, its projection, the residual):
        # sqrt(2 x 10) roundings of 2^-9 rms, with room of three
        err = (y.double() - ref).norm() / ref.norm()
        assert err <= 3 * 20 ** 0.5 * 2.0 ** -9, float(err)
        # every kept token behind the first step's, but the one that was changed, is the
        # model's choice
        choice = (y @ s.embed.t()).argmax(-1).tolist()
        start = x["kept"][0]
        wrong = [i for i in range(start, n) if x["tokens"][i] != choice[i - 1]]
        assert len(wrong) <= 1
    if nodes > 1:
        assert max(n for x in run for n in x["kept"][1:]) > 1
    # all pages are free again, each once
    assert (s.pool.shares == 0).all()
    head = int(s.head.item())
    assert head == 0 and sorted(s.pool.free_pages.tolist()) == list(range(s.pool.n_pages))
