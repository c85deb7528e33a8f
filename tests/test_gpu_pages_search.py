"""chimera_search_pages: candidates of the index, scores of the paged store, on
the tiny, 100k and 2M-long recipes, against the prune tap and 64-bit scores."""
import os

import numpy as np
import pytest
import torch

import synth
from paper_2608_23553_amd import ChimeraError, Pages, chimera
from util_build import product_builder
from util_gpu import q_tensor, say, setup
from util_pages import maxsim, mx_values, score_tolerance

pytestmark = pytest.mark.gpu


def _pages(c, k, skip=()):
    """A store of the corpus' documents but those of skip, and their values."""
    lens = np.diff(c.doc_off).astype(np.int32)
    x = synth.k_to_f32(k)
    v = mx_values(x)
    pg = Pages(int((-(-lens // 16)).sum()), len(lens) + 3, int(lens.max()))
    ids = np.setdiff1d(np.arange(len(lens)), skip)
    rows = np.concatenate([np.arange(c.doc_off[d], c.doc_off[d + 1]) for d in ids])
    pg.append(ids, torch.from_numpy(x[rows]).cuda(), lens[ids])
    docs = [v[c.doc_off[d]:c.doc_off[d + 1]] for d in range(len(lens))]
    for d in skip:
        docs[d] = docs[d][:0]
    return pg, docs


def _check(idx, pg, docs, qk, nprobe, ncand, k, label, dtype="bf16", queries=None):
    say("search_pages", label, qk.shape, nprobe, ncand, k)
    Q = q_tensor(qk, dtype)
    ids, scores = idx.search_pages(pg, Q, nprobe, ncand, k)
    cand, _, nval = idx.prune(Q, nprobe, ncand)
    torch.cuda.synchronize()
    ids, scores, cand, nval = (t.cpu().numpy() for t in (ids, scores, cand, nval))
    q64 = synth.k_to_f32(qk).astype(np.float64)
    for i in range(len(qk)) if queries is None else queries:
        kept = cand[i, :nval[i]]
        F = {int(d): maxsim(q64[i], docs[d]) for d in kept}
        # rounding of the sum, then of the key, then of the key's float
        tol = {d: score_tolerance(q64[i], docs[d]) + 2.0**-23 + 2.0**-24 * abs(F[d]) for d in F if F[d] > -np.inf}
        live = sorted(tol, key=lambda d: (-F[d], d))
        m = min(k, len(live))
        got = ids[i, :m]
        assert (ids[i, m:] == -1).all() and np.isneginf(scores[i, m:]).all(), label
        assert len(set(got)) == m and set(got) <= set(live), label
        for r in range(m):
            assert abs(scores[i, r] - F[got[r]]) <= tol[got[r]], (label, i, r, scores[i, r], F[got[r]])
        order = list(zip(-scores[i, :m], got))
        assert order == sorted(order), (label, i, "score descending, id ascending")
        if m < len(live):  # nothing left out is better than the last result
            assert max(F[d] - tol[d] for d in set(live) - set(got)) <= scores[i, m - 1] + 1e-12, (label, i)
    return ids


@pytest.mark.parametrize("name,ndocs,nq,k", [("tiny", None, 16, 10), ("100k", 6000, 5, 50), ("2m-long", 500, 3, 100)])
def test_search_from_pages(name, ndocs, nq, k):
    w, c, kk, cl, oi, idx = setup(name, ndocs)
    pg, docs = _pages(c, kk)
    q, src = c.queries(nq, w.Tq, query_seed=21)
    ncand = min(w.ncand, w.ndocs // 3)
    ids = _check(idx, pg, docs, q, w.nprobe, ncand, k, name)
    _check(idx, pg, docs, q[:2, :min(7, w.Tq)], w.nprobe, ncand, k, name + " f32, short queries", "f32")
    _check(idx, pg, docs, q[:1], w.nprobe, min(ncand, 100), 20, name + ", few candidates")
    assert np.mean(ids[:, 0] == src) >= 0.9  # the document that a query was drawn from comes first


def test_search_from_pages_in_sub_batches_with_documents_missing():
    """Documents that the store does not hold are left out; documents deleted from the index are no candidates."""
    w, c, kk, cl, oi, _ = setup("100k", 6000)
    idx = product_builder(c, w.nbits).upload(0)
    gone = np.arange(0, 6000, 3)
    pg, docs = _pages(c, kk, skip=gone)
    q, _ = c.queries(40, w.Tq, query_seed=22)
    old = os.environ.get("CHIMERA_SCRATCH_MB")
    os.environ["CHIMERA_SCRATCH_MB"] = "16"
    try:
        _check(idx, pg, docs, q, w.nprobe, 60, 50, "16 MB scratch", queries=(0, 1, 19, 39))
    finally:
        os.environ.pop("CHIMERA_SCRATCH_MB") if old is None else os.environ.__setitem__("CHIMERA_SCRATCH_MB", old)
    idx.delete(np.arange(1, 6000, 3))
    ids = _check(idx, pg, docs, q[:3], w.nprobe, 2000, 40, "deleted")
    assert (ids[ids >= 0] % 3 == 2).all()
    idx.close()


def test_search_from_pages_follows_the_store():
    """A store that changes between searches, on other streams than the searches."""
    w, c, kk, cl, oi, idx = setup("tiny")
    pg, docs = _pages(c, kk)
    q, src = c.queries(4, w.Tq, query_seed=23)
    s = torch.cuda.Stream()
    first = _check(idx, pg, docs, q, w.nprobe, w.ncand, 5, "before")
    best = np.unique(first[:, 0]).astype(np.int64)
    pg.drop(best, stream=s)
    for d in best:
        docs[d] = docs[d][:0]
    after = _check(idx, pg, docs, q, w.nprobe, w.ncand, 5, "dropped")
    assert not np.isin(after, best).any()


def test_search_from_pages_refusals():
    w, c, kk, cl, oi, idx = setup("tiny")
    q, _ = c.queries(2, w.Tq)
    Q = q_tensor(q, "bf16")
    small = Pages(4, 999, 32)
    pg = Pages(4, 1000, 32)
    ids = torch.full((2, 10), 7, dtype=torch.int32, device="cuda")
    sc = torch.full((2, 10), 3.0, device="cuda")
    for store, nprobe, ncand, k in ((small, 2, 256, 10), (pg, 0, 256, 10), (pg, 2, 5, 10)):
        with pytest.raises(ChimeraError) as e:
            idx.search_pages(store, Q, nprobe, ncand, k, out=(ids, sc))
        assert e.value.code == chimera.E_INVAL
    torch.cuda.synchronize()
    assert torch.all(ids == 7) and torch.all(sc == 3.0)
    idx.search_pages(pg, Q, 2, 256, 10, out=(ids, sc))
    assert torch.all(ids == -1) and torch.isneginf(sc).all()
