"""Calls on the paged store that its other tests do not make: a search where it
cannot be, tensors of another stream, another thread between two calls, queries
of any magnitude, plans that go round their buffers."""
import numpy as np
import pytest
import torch

from paper_2608_23553_amd import ChimeraError, Pages, chimera
from util_gpu import q_tensor, say, setup
from util_pages import check_scores, host, mx_values, same, tensor, units

pytestmark = pytest.mark.gpu


def _refused(code, f, *a, **k):
    with pytest.raises(ChimeraError) as e:
        f(*a, **k)
    assert e.value.code == code, e.value


# ------------------------------------------------------------ graphs
@pytest.mark.parametrize("before", ["nothing", "the null stream", "another stream"])
def test_a_search_in_a_capture_is_refused(before):
    """The capture goes on, the store and the index stay as they were, whatever work is queued on the store."""
    w, c, kk, cl, oi, idx = setup("tiny")
    q, _ = c.queries(2, w.Tq)
    Q = q_tensor(q, "bf16")
    rng = np.random.default_rng(31)
    pg = Pages(1000, 1000, 32)
    x = units(rng, 40)
    X, v = tensor(x), mx_values(x)
    own, out = Q[:, :8].float().contiguous(), torch.zeros(2, 1000, device="cuda")
    out_ids, out_scores = idx.search_pages(Pages(1, 1000, 1), Q, w.nprobe, w.ncand, 5)  # the index's scratch is there
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    docs = [v[:0]] * 1000
    if before != "nothing":
        pg.append([3, 4], X, [20, 20], stream=None if before == "the null stream" else side)
        docs[3], docs[4] = v[:20], v[20:]
    side.synchronize()
    say("capturing after", before)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _refused(chimera.E_UNSUPPORTED, idx.search_pages, pg, Q, w.nprobe, w.ncand, 5, out=(out_ids, out_scores))
        pg.score(own, out=out)
        _refused(chimera.E_UNSUPPORTED, idx.search_pages, pg, Q, w.nprobe, w.ncand, 5, out=(out_ids, out_scores))
    assert torch.all(out_ids == -1) and torch.isneginf(out_scores).all()
    for step in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, pg.score(own))
        check_scores(out[:, :6], own, docs, [range(6)] * 2, f"replay {step}")
        if step == 0:
            pg.append([5], X[:7], [7], stream=side)
            docs[5] = v[:7]
            side.synchronize()
            same(pg.read([5]), v[:7])
    pg.drop([3, 4, 5])
    assert pg.info()["ntokens"] == 0
