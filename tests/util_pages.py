"""The paged store's operators in 64 bits, for its tests: MXFP4 values, scores
and a store of plain arrays."""
import numpy as np
import torch

STEP = np.array([0.5, 0.5, 1.0, 2.0])  # spacing of the elements from 0, 1, 2, 4


def mx_values(x):
    """What MXFP4 makes of rows of 128 float values (float64, exact): NaN blocks where a value is not finite."""
    b = np.asarray(x, np.float64).reshape(-1, 4, 32)
    a = np.abs(b)
    bad = ~np.isfinite(b).all(-1)
    top = np.where(bad, 1.0, np.where(np.isfinite(a), a, 0).max(-1))
    e = np.frexp(top)[1] - 1                     # floor(log2), for 0: -1
    e = np.where(top < 2.0**-126, -127, e)       # exponent field 0
    scale = np.ldexp(1.0, np.maximum(e - 2, -127))[..., None]
    y = np.where(bad[..., None], 0.0, a) / scale
    step = np.where(y < 2, 0.5, np.where(y < 4, 1.0, 2.0))
    y = np.minimum(np.rint(y / step) * step, 6.0)
    v = np.copysign(y * scale, b)
    v[bad] = np.nan
    return v.reshape(-1, 128)


def grid(q):
    """Queries on the value grid: multiples of 2^-11 below 1/16, bfloat16 above."""
    q32 = torch.as_tensor(q).float().cpu()
    big = q32.to(torch.bfloat16).double().numpy()
    q64 = q32.double().numpy()
    return np.where(np.abs(q64) < 0.0625, np.rint(q64 * 2048) / 2048, big)


def maxsim(q, v):
    """Score of one query [Tq, 128] with one document's values [len, 128] (float64; NaN tokens never the best)."""
    v = v[~np.isnan(v).any(1)]
    return (q @ v.T).max(1).sum() if len(v) else -np.inf


def score_tolerance(q, v):
    """How far a float32 score may be off.  A query value is three digits of base 32, in magnitude at most |q| +
    2 * (512 + 16) / 2048 together; each of the 3 * 128 products is exact and each addition rounds by half a step of a
    partial sum of at most A = sum_i (|q_i| + 0.516) |v_i|; the Tq maxima are summed with at most Tq additions.  Query
    blocks of 8 or more lose up to 2^-15 of their largest value a component."""
    v = np.abs(v[~np.isnan(v).any(1)])
    if not len(v):
        return 0.0
    A = ((np.abs(q) + 0.516) @ v.T).max(1).sum()
    blocks = np.abs(q).reshape(len(q), 4, 32).max(-1)
    lost = np.where(blocks >= 8, blocks * 2.0**-15, 0.0).repeat(32, 1)
    return 2.0**-24 * (384 + len(q)) * A + (lost @ v.T).max(1).sum()


def units(rng, n):
    """Unit vectors, float32."""
    x = rng.standard_normal((n, 128))
    return (x / np.linalg.norm(x, axis=1, keepdims=True)).astype(np.float32)


def tensor(x, dtype="f32"):
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda()
    return t if dtype == "f32" else t.to(torch.bfloat16)


def host(t):
    return t.float().cpu().double().numpy()


def same(got, want, label=""):
    """Equal values, NaN for NaN."""
    got = host(got)
    assert got.shape == want.shape, f"{label}: {got.shape} != {want.shape}"
    bad = ~((got == want) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), f"{label}: {bad.sum()} values differ, first at {np.argwhere(bad)[0]}: " \
                          f"{got[bad][0]} for {want[bad][0]}"


def check_scores(got, Q, docs, lists, label=""):
    """got [nq, n] against documents docs[id] (values float64); lists [nq][n] ids, any outside: no document."""
    got = got.cpu().numpy()
    q = grid(Q)
    none = np.empty((0, 128))
    for i in range(len(q)):
        for c, d in enumerate(lists[i]):
            v = docs[d] if 0 <= d < len(docs) else none
            want, tol = maxsim(q[i], v), score_tolerance(q[i], v)
            ok = got[i, c] == want if not np.isfinite(want) else abs(got[i, c] - want) <= tol
            assert ok, f"{label}: query {i} entry {c} document {d}: {got[i, c]} for {want}, tolerance {tol}"
