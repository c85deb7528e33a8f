"""Calls on the paged store that its other tests do not make: a search where it
cannot be, tensors of another stream, another thread between two calls, queries
of any magnitude, plans that go round their buffers."""
import contextlib
import ctypes
import gc

import numpy as np
import pytest
import torch

import synth
from paper_2608_23553_amd import ChimeraError, Pages, chimera
from util_build import product_builder
from util_gpu import q_tensor, say, setup
from util_pages import check_scores, grid, host, mx_values, same, tensor, units

pytestmark = pytest.mark.gpu


def _refused(code, f, *a, **k):
    """Without a name that holds on to the error: its frames would keep a caller's graph until the next collection."""
    try:
        f(*a, **k)
    except ChimeraError as e:
        got, text = e.code, str(e)
    else:
        pytest.fail("not refused")
    assert got == code, text


@contextlib.contextmanager
def _nothing_collected():
    """Around a capture: a collection there may end the process, since a graph that it finds waits for the device, which
    a capture forbids."""
    gc.collect()
    gc.disable()
    try:
        yield
    finally:
        gc.enable()


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
    with _nothing_collected(), torch.cuda.graph(g):
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


def _hip():
    """The HIP runtime that torch has loaded."""
    with open("/proc/self/maps") as f:
        return ctypes.CDLL(next(line.split()[-1] for line in f if "libamdhip64" in line))


def test_calls_on_the_null_stream_while_a_blocking_stream_is_captured():
    """Work on the null stream would end such a capture: every call is refused and queues nothing, and all is well
    after it."""
    w, c, kk, cl, oi, idx = setup("tiny")
    q, _ = c.queries(2, w.Tq)
    Q = q_tensor(q, "bf16")
    rng = np.random.default_rng(32)
    x = units(rng, 50)
    X, v = tensor(x), mx_values(x)
    pg = Pages(1000, 1000, 64)
    pg.append([1, 2], X, [20, 30])
    out, rows = torch.full((2, 1000), 7.0, device="cuda"), torch.full((50, 128), 7.0, device="cuda")
    res = idx.search_pages(pg, Q, w.nprobe, w.ncand, 5)
    info, side = pg.info(), torch.cuda.Stream()
    torch.cuda.synchronize()
    H, s, g = _hip(), ctypes.c_void_p(), ctypes.c_void_p()
    assert torch.cuda.current_stream().cuda_stream == 0
    with _nothing_collected():
        assert H.hipStreamCreateWithFlags(ctypes.byref(s), 0) == 0 and H.hipStreamBeginCapture(s, 2) == 0
        try:
            for f in (lambda: pg.score(Q, out=out), lambda: pg.append([3], X, [50]), lambda: pg.drop([1]),
                      lambda: pg.read([1, 2], out=rows), lambda: pg.fork([1], [4]), lambda: pg.copy([1], [4]),
                      lambda: idx.search_pages(pg, Q, w.nprobe, w.ncand, 5, out=res),
                      # on another stream, which waits for the store's last work, on the null stream
                      lambda: pg.score(Q, out=out, stream=side), lambda: pg.append([3], X, [50], stream=side),
                      lambda: pg.drop([1], stream=side), lambda: pg.read([1, 2], out=rows, stream=side),
                      lambda: pg.fork([1], [4], stream=side), lambda: pg.copy([1], [4], stream=side),
                      lambda: idx.search_pages(pg, Q, w.nprobe, w.ncand, 5, out=res, stream=side)):
                _refused(chimera.E_UNSUPPORTED, f)
        finally:
            ended = H.hipStreamEndCapture(s, ctypes.byref(g))
    assert ended == 0 and H.hipGraphDestroy(g) == 0 and H.hipStreamDestroy(s) == 0
    torch.cuda.synchronize()
    assert torch.all(out == 7.0) and torch.all(rows == 7.0) and pg.info() == info
    same(pg.read([1, 2]), v)
    pg.score(Q, out=out, stream=side)
    side.synchronize()
    check_scores(out[:, :4], Q, [v[:0], v[:20], v[20:], v[:0]], [range(4)] * 2)


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


# ------------------------------------------------------------ queries of any magnitude
def _magnitudes(rng, n, lo=-12):
    """n queries [1, 128]: blocks whose largest values go from 2^lo to the largest of bfloat16, others down to 2^-19 of
    them."""
    q = rng.uniform(-1, 1, (n, 4, 32)) * 2.0 ** -rng.integers(0, 20, (n, 4, 32))
    q[:, :, rng.integers(0, 32)] = rng.uniform(1, 2, (n, 4))
    e = np.resize(np.arange(lo, 128), 4 * n).reshape(n, 4)
    return np.clip(q * 2.0 ** e[..., None], -3.38e38, 3.38e38).reshape(n, 1, 128).astype(np.float32)


def _lost(q):
    """How far the value used for a query value may be off [.., 128]: nothing below 8, above a half of a unit of which
    the block's largest value has 2^13 or more."""
    top = np.abs(q).reshape(*q.shape[:-1], 4, 32).max(-1)
    return np.where(top >= 8, top * 2.0**-14, 0.0).repeat(32, -1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", ["shared", "own lists", "one at a time"])
def test_query_values_of_every_magnitude(form, dtype):
    """Documents of one value 1: a score is the value used for the query's, which is a sum of a few exact terms."""
    rng = np.random.default_rng(61)
    eye = np.zeros((128, 128), np.float32)
    eye[np.arange(128), np.arange(128)] = 1
    pg = Pages(128, 128, 1)
    pg.append(np.arange(128), tensor(eye), [1] * 128)
    q = _magnitudes(rng, 140)
    q[0, 0, :5] = [8, 2.0**-11, 3 * 2.0**-11, 5, -7.96875]
    q[0, 0, 5:32] = 0
    Q = tensor(q, dtype)
    say("query values", form, dtype)
    if form == "own lists":
        got = pg.score(Q, torch.arange(128, dtype=torch.int32, device="cuda").repeat(len(q), 1))
    elif form == "shared":
        got = pg.score(Q)
    else:
        got = torch.cat([pg.score(x[None]) for x in Q])
    got, want = got.cpu().double().numpy(), grid(Q)[:, 0]
    off = np.abs(got - want)
    bad = ~(off <= _lost(want))
    assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], want[bad][:3])
    assert (got[np.abs(want).reshape(-1, 4, 32).max(-1).repeat(32, -1) < 8].size > 1000)


@pytest.mark.parametrize("e", [0, 3, 13, 60, 101, 102, 103, 106, 110, 117, 120, 125, 127])
@pytest.mark.parametrize("Tq", [5, 40])
def test_large_queries_and_small_documents(e, Tq):
    """Scores of ordinary size from queries up to the largest there are: all blocks of a query near 2^e, then only some."""
    rng = np.random.default_rng(62)
    x = rng.standard_normal((60, 128)) * 2.0**-e
    X = tensor(x)
    pg = Pages(6, 3, 30)
    pg.append([0, 1, 2], X, [10, 20, 30])
    v = mx_values(host(X))
    docs = [v[:10], v[10:30], v[30:]]
    q = rng.uniform(-1.98, 1.98, (3, Tq, 128)) * 2.0**e
    q[1, :, :64] *= 2.0**-e
    q[2, ::2] *= 2.0**-e
    Q = tensor(q)
    say("large queries", e, Tq)
    got = pg.score(Q).cpu().numpy()
    for i, g in enumerate(grid(Q)):
        top = np.abs(g).reshape(Tq, 4, 32).max(-1).repeat(32, -1)
        for d in range(3):
            a = np.abs(docs[d])
            # Each product is exact and each of 3 * 128 additions rounds by half a step of a partial sum.  The lower
            # digits are at most 2 * (512 + 16) units of 2^-11 below 8 (0.516), and of 2^-13 of the largest value above.
            A = ((np.abs(g) + np.maximum(0.516, 0.129 * top)) @ a.T).max(1).sum()
            tol = 2.0**-24 * (384 + Tq) * A + (_lost(g) @ a.T).max(1).sum()
            want = (g @ docs[d].T).max(1).sum()
            assert abs(got[i, d] - want) <= tol, (i, d, got[i, d], want, tol)


# ------------------------------------------------------------ views and plans
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("first", [1, 2, 4, 8, 31])
def test_rows_of_a_wider_tensor_at_any_offset(dtype, first):
    """Views whose rows begin at `first` of 192 values, padded and packed: what the library cannot take is copied."""
    rng = np.random.default_rng(71)
    lens = np.array([5, 0, 33, 40, 1], np.int32)
    wide = tensor(units(rng, 300).reshape(-1, 192), dtype).view(5, 40, 192)
    X = wide[..., first:first + 128]
    v = mx_values(host(X).reshape(-1, 128)).reshape(5, 40, 128)
    want = np.concatenate([v[i, :n] for i, n in enumerate(lens)])
    for name, t in (("padded", X), ("one document", X[3:4]), ("packed", wide.view(-1, 192)[:79, first:first + 128])):
        pg = Pages(20, 5, 40)
        if name == "padded":
            pg.append(np.arange(5), t, lens)
            same(pg.read(np.arange(5)), want, name)
        elif name == "one document":
            pg.append([2], t, [37])
            same(pg.read([2]), v[3, :37], name)
        else:
            pg.append(np.arange(5), t, lens)
            same(pg.read(np.arange(5)), v.reshape(-1, 128)[:79], name)


@pytest.mark.parametrize("n", [300, 3000])
def test_plans_that_go_round_their_buffers(n):
    """Plans of several times the buffers (half a MiB each), read in place (300 documents) and copied (3,000), on two
    streams and the null stream, with nothing waited for in between."""
    rng = np.random.default_rng(72)
    x = units(rng, 64)
    X, v = tensor(x), mx_values(x)
    pg = Pages(3 * n, 2 * n, 40)
    a, b = np.arange(n), np.arange(n, 2 * n)
    streams = [torch.cuda.Stream(), None, torch.cuda.Stream()]
    rows = torch.arange(n, device="cuda") % 64
    batches = [X.roll(k, 0)[rows] for k in range(5)]
    lists = [np.roll(v, k, 0)[np.arange(n) % 64] for k in range(5)]
    torch.cuda.synchronize()
    ones = np.ones(n, np.int32)
    rounds = -(-5 * (512 << 10) // (32 * 4 * n))  # each makes 4 plans of 32 bytes a document or more
    reads, wants = [], []
    for k in range(rounds):
        s = streams[k % 3]
        pg.drop(a, stream=s)
        pg.append(a, batches[k % 5], ones, stream=streams[(k + 1) % 3])
        pg.append(a, batches[(k + 1) % 5], ones, stream=s)
        pg.drop(b, stream=streams[(k + 2) % 3])
        pg.fork(a, b, 1 + (a + k) % 2, stream=s)
        if k % 8 == 7 or k == rounds - 1:
            reads.append(pg.read(np.stack([a, b], 1).reshape(-1), stream=streams[(k + 2) % 3]))
            both = np.stack([lists[k % 5], lists[(k + 1) % 5]], 1)
            wants.append(np.concatenate([r for i in range(n) for r in (both[i], both[i, :1 + (i + k) % 2])]))
    torch.cuda.synchronize()
    say("rounds", rounds, "reads", len(reads))
    for i, (r, want) in enumerate(zip(reads, wants)):
        same(r, want, f"read {i}")
