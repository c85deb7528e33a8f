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


# ------------------------------------------------------------ other threads
class _Between:
    """The library of a store; before each call but the first, `change` runs (another thread's call there)."""

    def __init__(self, library, change):
        self.library, self.change, self.calls = library, change, 0

    def __getattr__(self, name):
        def call(*a):
            self.calls += 1
            if self.calls > 1:
                self.change()
            return getattr(self.library, name)(*a)
        return call


@pytest.mark.parametrize("change", ["drop", "shorten", "extend", "nothing left", "from nothing"])
@pytest.mark.parametrize("given", [False, True])
def test_a_read_while_another_thread_changes_the_documents(change, given):
    """A read whose documents change between counting and reading is refused, and leaves what it was given alone."""
    rng = np.random.default_rng(51)
    x = units(rng, 90)
    X, v = tensor(x), mx_values(x)
    pg = Pages(12, 4, 60)
    empty = change == "from nothing"
    if not empty:
        pg.append([1, 2], X[:60], [40, 20])
    L, ids = pg._lib, np.array([1, 2], np.int64)

    def run():
        pg._lib = L
        if change == "drop":
            pg.drop([2])
        elif change == "nothing left":
            pg.drop([1, 2])
        elif change == "shorten":
            pg.copy([1], [1], [17])
        else:
            pg.append([2], X[60:69], [9])

    before = torch.full((0 if empty else 60, 128), 7.0, device="cuda")
    pg._lib = _Between(L, run)
    say("read while", change)
    _refused(chimera.E_INVAL, pg.read, ids, **({"out": before} if given else {}))
    pg._lib = L
    torch.cuda.synchronize()
    assert torch.all(before == 7.0)
    want = {"drop": [v[:40]], "nothing left": [v[:0]], "shorten": [v[:17], v[40:60]],
            "extend": [v[:60], v[60:69]], "from nothing": [v[60:69]]}[change]
    same(pg.read([1, 2]), np.concatenate(want))


def test_read_all_through_the_c_entry():
    import ctypes
    rng = np.random.default_rng(52)
    x = units(rng, 53)
    pg = Pages(5, 3, 33)
    pg.append([0, 1], tensor(x), [20, 33])
    L, h, ids, total = pg._lib, pg._h, (ctypes.c_int64 * 3)(1, 0, 2), ctypes.c_int64(-5)
    out, s = torch.full((60, 128), 7.0, device="cuda"), torch.cuda.current_stream().cuda_stream

    def read(n, rows, at=None):
        total.value = -5
        return L.chimera_pages_read_all(h, ids, n, out.data_ptr() if at is None else at, rows, chimera.F32,
                                        ctypes.byref(total), s), total.value

    assert read(3, -1, 0) == (0, 53) and read(1, -1, 0) == (0, 33) and read(0, -1, 0) == (0, 0)
    assert read(3, 54) == (chimera.E_INVAL, 53) and read(3, 52) == (chimera.E_INVAL, 53)
    assert read(3, 0) == (chimera.E_INVAL, 53) and read(3, 53, 0) == (chimera.E_INVAL, 53)
    ids[2] = 3
    assert read(3, 53) == (chimera.E_INVAL, -5)
    ids[2] = 2
    torch.cuda.synchronize()
    assert torch.all(out == 7.0)
    assert read(3, 53) == (0, 53)
    same(out[:53], mx_values(np.concatenate([x[20:], x[:20]])))
    assert torch.all(out[53:] == 7.0)
    assert L.chimera_pages_read(h, ids, 3, out.data_ptr(), 60, chimera.F32, s) == 0  # the other one takes more rows
    assert L.chimera_pages_read_all(h, ids, 3, out.data_ptr(), 53, chimera.F32, None, s) == chimera.E_INVAL
