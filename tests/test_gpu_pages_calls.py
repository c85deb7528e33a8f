"""Calls on the paged store that its other tests do not make: a search where it
cannot be, tensors of another stream, another thread between two calls, queries
of any magnitude, plans that go round their buffers."""
import numpy as np
import pytest
import torch

import synth
from paper_2608_23553_amd import ChimeraError, Pages, chimera
from util_build import product_builder
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


# ------------------------------------------------------------ streams
def _later(Q):
    """Q as a view that the library cannot take as it is."""
    wide = torch.zeros(Q.shape[0], Q.shape[1], 2, Q.shape[2], dtype=Q.dtype, device="cuda")
    wide[:, :, 0] = Q
    return wide[:, :, 0]


@pytest.mark.parametrize("call", ["search_pages", "search", "refine", "rabitq", "collab", "probe", "prune", "candidates"])
def test_a_search_on_another_stream_than_the_current_one(call):
    """Strided queries and new results of a call on a stream of its own, while the current stream has work to do and
    takes memory as soon as the call returns: the same as on the current stream."""
    w, c, kk, cl, oi, idx = setup("tiny")
    if call in ("rabitq", "collab"):
        signs = synth.rotation_signs(17) if call == "rabitq" else None
        idx = product_builder(c, w.nbits, rabitq_signs=signs).upload(0)
        if call == "collab":
            idx.attach_fullbit(synth.k_to_bf16_bits(kk))
    q, _ = c.queries(16, w.Tq, query_seed=41)
    Q = q_tensor(q, "bf16")
    pg = Pages(4000, 1000, 64)
    lens = np.diff(c.doc_off).astype(np.int32)
    pg.append(np.arange(len(lens)), torch.from_numpy(synth.k_to_f32(kk)).cuda(), lens)
    args = (w.nprobe, w.ncand, 10)
    f = {"search_pages": lambda Q, **k: idx.search_pages(pg, Q, *args, **k),
         "search": lambda Q, **k: idx.search(Q, *args, **k),
         "refine": lambda Q, **k: idx.search(Q, *args, refine=chimera.REFINE_TOKEN, **k),
         "rabitq": lambda Q, **k: idx.search_rabitq(Q, *args, **k),
         "collab": lambda Q, **k: idx.search_collab(Q, w.nprobe, w.ncand, 20, 2, 10, **k),
         "probe": lambda Q, **k: idx.probe(Q, w.nprobe, **k),
         "prune": lambda Q, **k: idx.prune(Q, w.nprobe, w.ncand, **k),
         "candidates": lambda Q, **k: idx.candidates(Q, w.nprobe, **k)}[call]
    want = f(Q)
    view = _later(Q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        say(call, "beside the current stream")
        torch.cuda._sleep(20_000_000)
        got = f(view, stream=side)
        junk = [torch.full((n,), float("nan"), device="cuda") for n in (160, 16 * 32 * 64, 1 << 18) for _ in range(4)]
        side.synchronize()
        torch.cuda.synchronize()
        for a, b in zip(_written(call, got), _written(call, want)):
            assert type(a) is type(b) and a.shape == b.shape and bool((a == b).all()), call
        del got, junk


def _written(call, out):
    """What a call writes of its outputs."""
    if call == "candidates":
        offsets, docs = out
        return offsets, docs[:int(offsets[-1])]
    if call == "prune":
        cand, keys, n = out
        here = torch.arange(cand.shape[1], device="cuda") < n[:, None]
        return cand[here], keys[here], n
    return out
