"""The paged MXFP4 store on the GPU against the same in 64 bits: quantising and
reading back bit for bit, scores within the rounding of float32 sums, sharing,
copying and dropping against plain lists, streams, graphs, refusals."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2608_23553_amd import ChimeraError, Pages, chimera
from util_gpu import say
from util_pages import check_scores, grid, host, maxsim, mx_values, same, tensor, units

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _filled(rng, lens, dtype="f32", spare=0, **kw):
    """A store with documents of these lengths, and their values."""
    lens = np.asarray(lens, np.int32)
    npages = int((-(-lens.astype(np.int64) // 16)).sum()) + spare
    pg = Pages(max(npages, 1), len(lens), max(int(lens.max(initial=1)), 1), **kw)
    X = tensor(units(rng, int(lens.sum())), dtype)
    pg.append(np.arange(len(lens)), X, lens)
    v, off = mx_values(host(X)), np.concatenate([[0], np.cumsum(lens)])
    return pg, [v[a:b] for a, b in zip(off, off[1:])]


# ------------------------------------------------------------ quantising
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens", [[1], [16], [15, 17, 1, 0, 32, 33], [256, 257, 1000], [0, 0], list(range(64))])
def test_append_and_read_are_exact(dtype, lens):
    rng = np.random.default_rng(len(lens))
    say("append", dtype, lens[:6])
    pg, docs = _filled(rng, lens, dtype)
    ids = rng.permutation(len(lens))
    want = np.concatenate([docs[i] for i in ids]) if len(lens) else np.empty((0, 128))
    same(pg.read(ids), want, "bf16")
    same(pg.read(ids, dtype=torch.float32), want, "f32")
    assert np.array_equal(pg.lengths(), lens) and pg.info()["ntokens"] == sum(lens)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_exponent_border_and_special_value(dtype):
    """Blocks of every scale, elements at and next to the borders between two codes, zeros, subnormals, the largest
    finite values, infinities and NaN."""
    rng = np.random.default_rng(3)
    borders = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    b32 = borders.astype(np.float32)
    near = np.concatenate([borders, np.nextafter(b32, 9), np.nextafter(b32, 0)])
    rows = []
    for e in range(-149, 128):
        m = rng.uniform(4, 8, (4, 32)) * rng.choice([-1, 1], (4, 32))
        m[:, 1:22] = near
        m[:, 22:] *= 2.0 ** -rng.integers(0, 9, (4, 10))
        m[:, 0] = [4, 6, 7.99, -5]
        rows.append(np.clip(np.ldexp(m, min(e - 2, 125)), -3.4e38, 3.4e38))
    x = np.stack(rows).astype(np.float32).reshape(-1, 128)
    z = np.zeros((7, 128), np.float32)
    z[1] = -0.0
    z[2, 5] = np.inf
    z[3, 40] = -np.inf
    z[4, 127] = np.nan
    z[5] = np.nan
    z[6, 64:] = 1.0
    z[6, 0] = np.float32(1e-45)
    x = np.concatenate([x, z, z[::-1]])
    X = tensor(x, dtype)
    pg = Pages(-(-len(x) // 16), 1, len(x))
    pg.append([0], X, [len(x)])
    want = mx_values(host(X))
    assert np.isnan(want).any() and (np.abs(want[np.isfinite(want)]) > 1e38).any()
    same(pg.read([0], dtype=torch.float32), want, "f32")
    same(pg.read([0]), want, "bf16")


def test_token_by_token_and_across_pages():
    rng = np.random.default_rng(5)
    x = units(rng, 3 * 70)
    v = mx_values(x).reshape(3, 70, 128)
    X = tensor(x).view(3, 70, 128)
    pg = Pages(15, 4, 70)
    have = 0
    for step in [1] * 20 + [15, 1, 16, 17, 1]:
        pg.append([2, 0, 3], X[:, have:have + step].contiguous())
        have += step
        same(pg.read([2, 0, 3]), v[:, :have].reshape(-1, 128), f"{have} tokens")
    assert have == 70 and pg.info()["free_pages"] == 0 and pg.lengths().tolist() == [70, 0, 70, 70]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_padded_strided_and_unaligned_tensors(dtype):
    rng = np.random.default_rng(6)
    lens = np.array([5, 0, 33, 40, 1], np.int32)
    x = units(rng, 5 * 40).reshape(5, 40, 128)
    X = tensor(x.reshape(-1, 128), dtype).view(5, 40, 128)
    want = np.concatenate([mx_values(host(X[i, :n])) for i, n in enumerate(lens)])
    X = X.clone()
    for i, n in enumerate(lens):
        X[i, n:] = float("nan")  # what stands behind a document is not read
    wide = torch.full((5, 40, 192), float("nan"), dtype=DT[dtype], device="cuda")
    wide[..., 32:160] = X
    flat = torch.zeros(5 * 40 * 128 + 1, dtype=DT[dtype], device="cuda")
    flat[1:] = X.flatten()
    swapped = X.transpose(0, 1).contiguous().transpose(0, 1)
    for name, t in (("padded", X), ("wide rows", wide[..., 32:160]), ("unaligned", flat[1:].view(5, 40, 128)),
                    ("token-major", swapped), ("odd offset", wide[..., 31:159].roll(-1, -1))):
        pg = Pages(20, 5, 40)
        pg.append(np.arange(5), t if name != "odd offset" else wide[..., 32:160], lens)
        same(pg.read(np.arange(5)), want, name)
    packed = torch.cat([wide[i, :n, 32:160] for i, n in enumerate(lens)])
    rows = torch.empty(2 * len(packed), 128, dtype=DT[dtype], device="cuda")
    rows[::2] = packed
    pg = Pages(20, 5, 40)
    pg.append(np.arange(5), rows[::2], lens)
    same(pg.read(np.arange(5)), want, "every other row")


# ------------------------------------------------------------ scores
@pytest.mark.parametrize("Tq", [1, 2, 16, 31, 32, 33, 48, 64])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_of_every_query_length(Tq, dtype):
    rng = np.random.default_rng(Tq)
    lens = [1, 0, 2, 15, 16, 17, 31, 32, 33, 47, 64, 65, 100, 180, 512, 700]
    pg, docs = _filled(rng, lens, dtype)
    Q = tensor(units(rng, 3 * Tq), dtype).view(3, Tq, 128)
    say("score", Tq, dtype)
    check_scores(pg.score(Q), Q, docs, [range(len(lens))] * 3, "all")
    lists = np.array([rng.integers(0, len(lens), 21) for _ in range(3)], np.int32)
    lists[1, 3], lists[1, 4], lists[2, 0], lists[0, 20] = -1, len(lens), -2**31, 2**31 - 1
    ids = torch.from_numpy(lists).cuda()
    check_scores(pg.score(Q, ids), Q, docs, lists, "lists")
    check_scores(pg.score(Q, ids[1]), Q, docs, [lists[1]] * 3, "one list")
    check_scores(pg.score(Q, ids[:, 2:9]), Q, docs, lists[:, 2:9], "part of a list")
    check_scores(pg.score(Q, ids[:, ::3]), Q, docs, lists[:, ::3], "every third")
    check_scores(pg.score(Q[1:2], ids[1:2, 5:6]), Q[1:2], docs, lists[1:2, 5:6], "one")


@pytest.mark.parametrize("n,nq", [(1, 1), (3, 70), (257, 9), (2000, 2), (999, 33), (2, 3001), (256, 1), (85, 3)])
def test_scores_of_many_documents(n, nq):
    rng = np.random.default_rng(n)
    pg, docs = _filled(rng, rng.integers(0, 40, n), "bf16")
    Q = tensor(units(rng, nq * 32), "bf16").view(nq, 32, 128)
    say("score", n, nq)
    got = pg.score(Q)
    check_scores(got, Q[:2], docs, [range(n)] * 2, "first")
    check_scores(got[-1:], Q[-1:], docs, [range(n)], "last")
    lists = torch.from_numpy(np.stack([rng.permutation(n) for _ in range(nq)]).astype(np.int32)).cuda()
    assert torch.equal(pg.score(Q, lists), torch.gather(got, 1, lists.long()))


@pytest.mark.parametrize("pattern", [[0, 6], [0, 0, 17, 0], [6, 0], [0, 40], [5, 6], [16, 0, 16], [1]])
def test_empty_documents_between_others(pattern):
    """Lists long enough that a wave takes several entries: one list for many queries, a list each, and one query."""
    rng = np.random.default_rng(7)
    pg, docs = _filled(rng, pattern * (1000 // len(pattern)), "bf16")
    n = len(docs)
    Q = tensor(units(rng, 41 * 20), "bf16").view(41, 20, 128)
    got = pg.score(Q)
    check_scores(got[:1], Q[:1], docs, [range(n)], "one list")
    assert torch.equal(got, torch.cat([pg.score(q[None]) for q in Q]))
    lists = torch.arange(n, dtype=torch.int32, device="cuda").repeat(41, 1)
    assert torch.equal(got, pg.score(Q, lists))
    assert torch.equal(got.flip(1)[:, 7:], pg.score(Q, lists.flip(1)[:, 7:]))


@pytest.mark.parametrize("nq", [2, 5, 16, 33, 130])
@pytest.mark.parametrize("Tq", [1, 2, 3, 4, 5, 8, 9, 16, 17])
def test_short_queries_that_share_a_list(Tq, nq):
    """Many queries side by side score as each does alone: also with one that has large values or none that are finite
    among them, empty documents, and entries that name no document."""
    rng = np.random.default_rng(100 * Tq + nq)
    pg, docs = _filled(rng, rng.integers(0, 40, 90), "bf16")
    q = units(rng, nq * Tq).reshape(nq, Tq, 128)
    Q = tensor(q)
    ids = rng.integers(-3, 93, 330).astype(np.int32)
    one = torch.from_numpy(ids).cuda()
    each = one.expand(nq, 330).contiguous()
    say("score", Tq, nq)
    got = pg.score(Q, one)
    check_scores(torch.cat([got[:1], got[-1:]]), torch.cat([Q[:1], Q[-1:]]), docs, [ids] * 2, "first and last")
    assert torch.equal(got, pg.score(Q, each)) and torch.equal(got, pg.score(Q, one.expand(nq, 330)))
    overlapping = one.as_strided((nq, 100), (1, 1))
    assert torch.equal(pg.score(Q, overlapping)[-1], got[-1, nq - 1:nq + 99])
    Q[nq // 2, Tq // 2, 5:70] = 3000.0
    Q[nq - 1, 0, 127] = float("nan")
    mixed = pg.score(Q, one)
    finite = [i for i in range(nq) if i not in (nq // 2, nq - 1)]
    assert torch.equal(mixed[finite], got[finite])
    if nq > 2:
        check_scores(mixed[nq // 2:nq // 2 + 1], Q[nq // 2:nq // 2 + 1], docs, [ids], "large values")
    own = pg.score(Q, each)
    assert torch.equal(mixed.nan_to_num(nan=9e9), own.nan_to_num(nan=9e9))


@pytest.mark.parametrize("Tq", [1, 3, 8, 11, 32])
def test_a_long_list_that_short_queries_share(Tq):
    """Waves that take 64 entries each."""
    rng = np.random.default_rng(Tq)
    pg, docs = _filled(rng, rng.integers(0, 20, 300), "bf16")
    Q = tensor(units(rng, 70 * Tq), "bf16").view(70, Tq, 128)
    ids = torch.from_numpy(rng.integers(-3, 310, 140_000).astype(np.int32)).cuda()
    say("score", Tq)
    all_docs = torch.cat([pg.score(Q[i:i + 1]) for i in range(70)])
    want = torch.where((ids >= 0) & (ids < 300), all_docs[:, ids.clamp(0, 299).long()], -float("inf"))
    assert torch.equal(pg.score(Q, ids), want)


def test_queries_as_views():
    """Queries that are strided, transposed or not 16-byte aligned, and repeated documents in a read."""
    rng = np.random.default_rng(18)
    pg, docs = _filled(rng, [20, 0, 70])
    q = tensor(units(rng, 3 * 5 * 2), "bf16").view(3, 10, 128)
    flat = torch.zeros(3 * 10 * 128 + 3, dtype=torch.bfloat16, device="cuda")
    flat[3:] = q.flatten()
    for name, Q in (("every other token", q[:, ::2]), ("some queries", q[::2]), ("token-major", q.transpose(0, 1)),
                    ("unaligned", flat[3:].view(3, 10, 128)), ("one", q[1:2, 9:])):
        check_scores(pg.score(Q), Q, docs, [range(3)] * len(Q), name)
    same(pg.read([2, 0, 1, 2]), np.concatenate([docs[2], docs[0], docs[2]]))


@pytest.mark.parametrize("Tq", [20, 50])
def test_few_long_documents(Tq):
    """Few entries: four waves share each document, whose pages do not divide evenly."""
    rng = np.random.default_rng(Tq)
    lens = [1, 15, 16, 17, 33, 48, 49, 64, 65, 0, 1023, 1024, 1041, 5000]
    pg, docs = _filled(rng, lens, "bf16")
    Q = tensor(units(rng, 2 * Tq)).view(2, Tq, 128)
    check_scores(pg.score(Q), Q, docs, [range(len(lens))] * 2, "few")
    many = torch.arange(len(lens), dtype=torch.int32, device="cuda").repeat(40)
    assert torch.equal(pg.score(Q, many)[:, -len(lens):], pg.score(Q))


def test_values_that_are_not_finite_never_win():
    rng = np.random.default_rng(8)
    x = units(rng, 5 * 50).reshape(5, 50, 128)
    x[0, ::2, 3] = np.nan         # every other token
    x[1, :, 64] = np.inf          # all tokens
    x[2, 49, 127] = -np.inf       # the last token
    x[3, 0] = np.nan
    X = tensor(x.reshape(-1, 128))
    pg = Pages(20, 5, 50)
    pg.append(np.arange(5), X, [50] * 5)
    docs = list(mx_values(host(X)).reshape(5, 50, 128))
    Q = tensor(np.concatenate([x[0, 0:1], units(rng, 20)])[1:]).view(1, 20, 128)
    got = pg.score(Q)
    check_scores(got, Q, docs, [range(5)])
    assert got[0, 1] == -np.inf and torch.isfinite(got[0, [0, 2, 3, 4]]).all()


@pytest.mark.parametrize("scale", [2.0**-12, 0.01, 0.24, 0.26, 0.499, 0.502, 1.0, 3.0, 7.9, 8.1, 1000.0, 1e30])
def test_queries_and_documents_of_any_size(scale):
    """Query values below and above 8, and documents scaled the other way."""
    rng = np.random.default_rng(9)
    x = rng.standard_normal((60, 128)) * 2.0 ** rng.integers(-6, 6, (60, 1))
    X = tensor(np.clip(x / scale, -1e37, 1e37))
    pg = Pages(6, 3, 30)
    pg.append([0, 1, 2], X, [10, 20, 30])
    v = mx_values(host(X))
    Q = tensor(rng.uniform(-1, 1, (2 * 7, 128)) * scale).view(2, 7, 128)
    docs = [v[:10], v[10:30], v[30:]]
    check_scores(pg.score(Q), Q, docs, [range(3)] * 2, f"scale {scale}")


def test_every_query_value_below_a_half_and_some_above():
    """One-hot documents of value 1: the score is the query value itself, exactly, in blocks whose largest value is up
    to 1/2 and beyond (two digits and three)."""
    k = np.arange(0, 4096, dtype=np.float64) / 2048
    bf = torch.from_numpy(k).to(torch.bfloat16).double().numpy()
    k = k[(k < 0.0625) | (k == bf)]                    # the grid
    k = np.concatenate([k, -k])
    eye = np.zeros((128, 128), np.float32)
    eye[np.arange(128), np.arange(128)] = 1
    X = tensor(eye)
    pg = Pages(128, 128, 1)
    pg.append(np.arange(128), X, [1] * 128)
    for most in (0.25, 0.5, 2.0):
        v = k[np.abs(k) <= most]
        v = np.resize(v, -(-len(v) // 128) * 128).reshape(-1, 1, 128)
        for order in (v, np.random.default_rng(0).permuted(v.reshape(-1)).reshape(v.shape)):
            got = pg.score(torch.from_numpy(order).float().cuda())
            assert np.array_equal(got.cpu().numpy(), order[:, 0]), most


def test_unit_vectors_score_to_the_last_bit():
    """Products of unit vectors on the grid are sums of few bits: the float32 score is the rounded 64-bit one."""
    rng = np.random.default_rng(10)
    pg, docs = _filled(rng, [40] * 30)
    Q = torch.from_numpy(grid(units(rng, 32))).float().cuda().view(1, 32, 128)
    got = pg.score(Q).cpu().numpy()[0]
    q = grid(Q)[0]
    for d in range(30):
        want = maxsim(q, docs[d])
        # 32 additions of float32 values below 32: each rounds by at most 2^-20
        assert abs(got[d] - want) <= 32 * 2.0**-20


# ------------------------------------------------------------ sharing, copying, dropping
def test_random_calls_against_plain_lists():
    rng = np.random.default_rng(11)
    ndocs, max_len = 14, 90
    stores = [Pages(45, ndocs, max_len), Pages(30, ndocs, max_len)]
    plain = [[np.empty((0, 128))] * ndocs for _ in stores]
    refused = done = 0
    for call in range(260):
        k = int(rng.integers(0, 2))
        pg, docs = stores[k], plain[k]
        n = int(rng.integers(1, 6))
        ids = rng.permutation(ndocs)[:n]
        what = rng.choice(["append", "append", "fork", "copy", "self", "drop"])
        before = [list(p) for p in plain]
        try:
            if what == "append":
                lens = rng.integers(0, 45, n)
                X = tensor(units(rng, int(lens.sum())), rng.choice(["f32", "bf16"]))
                pg.append(ids, X, lens)
                parts = np.split(mx_values(host(X)), np.cumsum(lens)[:-1])
                for d, p in zip(ids, parts):
                    docs[d] = np.concatenate([docs[d], p])
            elif what == "fork":
                src = rng.integers(0, ndocs, n)
                lens = np.array([rng.integers(0, len(docs[d]) + 1) for d in src])
                pg.fork(src, ids, lens)
                for s, d, m in zip(src, ids, lens):
                    docs[d] = before[k][s][:m]
            elif what == "drop":
                pg.drop(np.concatenate([ids, ids[:1]]))
                for d in ids:
                    docs[d] = np.empty((0, 128))
            else:
                t = k if what == "self" else int(rng.integers(0, 2))
                src = ids if what == "self" else rng.integers(0, ndocs, n)
                pos = [np.flatnonzero(rng.random(len(docs[d])) < rng.choice([0.1, 0.6, 1.0])) for d in src]
                pg.copy(src, ids, [len(p) for p in pos], np.concatenate(pos), to=stores[t])
                for s, d, p in zip(src, ids, pos):
                    plain[t][d] = before[k][s][p]
            done += 1
        except ChimeraError as e:
            assert e.code in (chimera.E_INVAL, chimera.E_NOMEM), (call, what, e)
            plain = before
            refused += 1
        if call % 10 == 9 or call > 240:
            for pg, docs in zip(stores, plain):
                assert np.array_equal(pg.lengths(), [len(d) for d in docs]), (call, what)
                same(pg.read(np.arange(ndocs)), np.concatenate(docs), f"call {call} {what}")
    assert done > 80 and refused > 10
    Q = tensor(units(rng, 2 * 9)).view(2, 9, 128)
    for pg, docs in zip(stores, plain):
        check_scores(pg.score(Q), Q, docs, [range(ndocs)] * 2, "after random calls")
        pg.drop(np.arange(ndocs))
        assert pg.info()["free_pages"] == pg.info()["npages"] and pg.info()["ntokens"] == 0
        assert torch.all(torch.isneginf(pg.score(Q)))


def test_a_revision_shares_its_prefix():
    """Fork, append to both, compact one, drop the other: each document reads and scores as its own list."""
    rng = np.random.default_rng(12)
    pg = Pages(16, 3, 120)
    x = units(rng, 160)
    v = mx_values(x)
    pg.append([0], tensor(x[:100]), [100])
    free = pg.info()["free_pages"]
    pg.fork([0], [1], [70])
    assert free - pg.info()["free_pages"] == 1  # four whole pages shared, six tokens copied
    pg.append([1, 0], tensor(np.concatenate([x[100:130], x[130:140]])), [30, 10])
    docs = [np.concatenate([v[:100], v[130:140]]), np.concatenate([v[:70], v[100:130]]), v[:0]]
    same(pg.read([0, 1]), np.concatenate(docs[:2]))
    keep = np.flatnonzero(rng.random(110) < 0.4)
    pg.copy([0], [0], [len(keep)], keep)
    docs[0] = docs[0][keep]
    same(pg.read([1, 0]), np.concatenate([docs[1], docs[0]]))
    Q = tensor(units(rng, 32)).view(1, 32, 128)
    check_scores(pg.score(Q), Q, docs, [range(3)])
    pg.drop([1])
    same(pg.read([0]), docs[0])
    assert pg.info()["free_pages"] == 16 - -(-len(keep) // 16)


def test_long_document_and_offsets_past_32_bits():
    """Documents of the largest length until the pool's last page starts above 2^32 bytes."""
    rng = np.random.default_rng(13)
    n = 1 << 20
    ndocs = 62
    pg = Pages(ndocs * (n // 16) + 1, ndocs + 1, n)
    X = tensor(units(rng, 4096), "bf16").repeat(n // 4096, 1)
    v = mx_values(host(X[:4096]))
    for d in range(ndocs):
        pg.append([d], X, [n])
    pg.append([ndocs], X[5:12], [7])
    assert pg.info()["npages"] * 1088 > 2**32 and pg.info()["free_pages"] == 0
    same(pg.read([ndocs]), v[5:12])
    say("reading the last long document")
    got = pg.read([ndocs - 1])
    same(got[:4096], v), same(got[-4096:], v)
    Q = tensor(units(rng, 8), "bf16").view(1, 8, 128)
    ids = torch.tensor([ndocs, ndocs - 1, 0], dtype=torch.int32, device="cuda")
    say("scoring long documents")
    check_scores(pg.score(Q, ids), Q, [v[5:12], v, v], [range(3)])
    pg.drop([0])
    pg.copy([ndocs - 1], [0], [3], [0, 4097, n - 1])
    same(pg.read([0]), v[[0, 1, 4095]])


# ------------------------------------------------------------ streams and graphs
def test_calls_on_different_streams_follow_one_another():
    rng = np.random.default_rng(14)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    x = units(rng, 60 * 200)
    X = tensor(x)
    v = mx_values(x).reshape(200, 60, 128)
    Q = tensor(units(rng, 32)).view(1, 32, 128)
    back = X.flip(0)
    torch.cuda.synchronize()
    pg = Pages(200 * 7, 400, 64)
    pg.append(np.arange(200), X, [60] * 200, stream=s1)
    a = pg.score(Q, stream=s2)
    pg.fork(np.arange(200), np.arange(200, 400), [33] * 200, stream=s1)
    pg.drop(np.arange(200), stream=s2)
    b = pg.score(Q)
    pg.append(np.arange(200), back, [60] * 200, stream=s2)
    c = pg.read(np.arange(400), stream=s1)
    torch.cuda.synchronize()
    check_scores(a[:, :200], Q, list(v), [range(200)], "first")
    assert torch.isneginf(a[:, 200:]).all() and torch.isneginf(b[:, :200]).all()
    check_scores(b[:, 200:], Q, [d[:33] for d in v], [range(200)], "forked")
    same(c, np.concatenate([mx_values(x[::-1]), v[:, :33].reshape(-1, 128)]), "last")


def test_score_in_a_graph():
    """A captured score, replayed between changes of the store; the calls that cannot be captured say so."""
    rng = np.random.default_rng(15)
    pg, docs = _filled(rng, [20, 40, 60, 0], spare=20)
    Q = tensor(units(rng, 2 * 24)).view(2, 24, 128)
    ids = torch.tensor([[3, 1, 2], [0, 0, 3]], dtype=torch.int32, device="cuda")
    out = torch.zeros(2, 3, device="cuda")
    X = tensor(units(rng, 9))
    pg.score(Q, ids, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pg.score(Q, ids, out=out)
        for call in (lambda: pg.append([3], X, [9]), lambda: pg.drop([0]), lambda: pg.fork([0], [3]),
                     lambda: pg.copy([0], [3]), lambda: pg.read([0], out=torch.empty_like(X).resize_(20, 128))):
            with pytest.raises(ChimeraError) as e:
                call()
            assert e.value.code == chimera.E_UNSUPPORTED
    lists = ids.cpu().numpy()
    for step in range(4):
        out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        check_scores(out, Q, docs, lists, f"replay {step}")
        assert torch.equal(out, pg.score(Q, ids))
        if step == 0:
            pg.append([3], X, [9])
            docs[3] = mx_values(host(X))
        elif step == 1:
            pg.drop([1])
            docs[1] = docs[1][:0]
        else:
            Q.copy_(torch.roll(Q, 1, 0))
        torch.cuda.synchronize()


def test_more_queries_than_one_launch_takes():
    """300,000 documents of one token: a launch takes 1,786 queries with a list each, and as many groups of them."""
    rng = np.random.default_rng(19)
    n, nq = 300_000, 1790
    X = tensor(units(rng, 5000), "bf16").repeat(n // 5000, 1)
    pg = Pages(n, n, 1)
    pg.append(np.arange(n), X, np.ones(n, np.int32))
    Q = tensor(units(rng, nq), "bf16").view(nq, 1, 128)
    got = pg.score(Q)
    for q in (0, 1, 1785, 1786, 1789):
        assert torch.equal(got[q], pg.score(Q[q:q + 1])[0]), q
    ids = torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda").expand(nq, n)
    own = pg.score(Q, ids.contiguous())
    assert torch.equal(own, got.flip(1))
    assert torch.equal(pg.score(Q, ids), own)  # expanded: one list
    v = mx_values(host(X[:5000]))
    check_scores(got[:2, :5000], Q[:2], [t[None] for t in v], [range(5000)] * 2)
    del got, own
    Q = tensor(units(rng, 3575 * 17), "bf16").view(3575, 17, 128)
    got = pg.score(Q)  # two queries a group
    for q in (0, 3571, 3572, 3574):
        assert torch.equal(got[q], pg.score(Q[q:q + 1])[0]), q


def test_two_host_threads():
    """Calls of two threads on one store: each is done or refused as busy, and the store stays whole."""
    import threading
    rng = np.random.default_rng(20)
    x = units(rng, 64)
    X, v = tensor(x), mx_values(x)
    pg = Pages(4000, 2000, 64)
    a, b = np.arange(1000), np.arange(1000, 2000)
    lens = np.ones(1000, np.int32)
    one = X[:1].expand(1000, 128).contiguous()
    errors = []

    def work(ids):
        done = 0
        for _ in range(400):
            try:
                pg.append(ids, one, lens)
                done += 1
            except ChimeraError as e:
                if e.code != chimera.E_BUSY:
                    errors.append(e)
            if done == 5:
                break
        counts.append(done)

    counts = []
    threads = [threading.Thread(target=work, args=(ids,)) for ids in (a, b)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors and all(counts)
    got = pg.lengths()
    assert sorted({tuple(set(got[:1000])), tuple(set(got[1000:]))}) == sorted({(c,) for c in counts})
    same(pg.read([0, 1999]), np.repeat(v[:1], got[0] + got[1999], 0))


def test_many_calls_without_waiting():
    """More calls under way than plan buffers, over several stores."""
    rng = np.random.default_rng(16)
    x = units(rng, 100)
    X, v = tensor(x), mx_values(x)
    stores = [Pages(8, 2, 100) for _ in range(3)]
    for i in range(120):
        pg = stores[i % 3]
        pg.drop([0, 1])
        pg.append([0], X[:50 + i % 7], [50 + i % 7])
        pg.fork([0], [1], [40])
    for k, pg in enumerate(stores):
        m = 50 + (117 + k) % 7
        same(pg.read([0, 1]), np.concatenate([v[:m], v[:40]]), f"store {k}")


# ------------------------------------------------------------ refusals
def test_refusals_leave_everything_as_it_was():
    rng = np.random.default_rng(17)
    pg, docs = _filled(rng, [20, 33, 0, 0, 0], spare=3)
    x = units(rng, 64)
    X = tensor(x)
    info, Q = pg.info(), tensor(x[:32]).view(1, 32, 128)

    def refused(code, f, *a, **k):
        with pytest.raises(ChimeraError) as e:
            f(*a, **k)
        assert e.value.code == code, e.value

    bad, nomem = chimera.E_INVAL, chimera.E_NOMEM
    refused(bad, pg.append, [5], X[:1], [1])
    refused(bad, pg.append, [-1], X[:1], [1])
    refused(bad, pg.append, [2, 2], X[:2], [1, 1])
    refused(bad, pg.append, [1], X[:1], [1])            # max_len is 33
    refused(bad, pg.append, [2], X[:1, :64], [1])       # half a token
    refused(nomem, pg.append, [2, 3], X[:64], [32, 32])
    refused(bad, pg.fork, [0], [1])
    refused(bad, pg.fork, [0], [2], [21])
    refused(bad, pg.fork, [0, 1], [2, 2])
    refused(bad, pg.fork, [0, 2], [2, 3])
    refused(bad, pg.fork, [7], [2])
    refused(nomem, pg.copy, [1, 0], [2, 3])
    refused(bad, pg.copy, [0], [2], [2], [1, 1])
    refused(bad, pg.copy, [0], [2], [1], [20])
    refused(bad, pg.copy, [0], [2], [1], [-1])
    refused(bad, pg.copy, [0, 0], [0, 2], [1, 1])
    refused(bad, pg.drop, [0, 5])
    refused(bad, pg.read, [0, 5])
    refused(bad, pg.lengths, [-1])
    small = Pages(4, 2, 16)
    refused(bad, pg.copy, [0], [0], to=small)           # longer than its documents can be
    refused(chimera.E_UNSUPPORTED, pg.score, tensor(units(rng, 65)).view(1, 65, 128))
    refused(bad, pg.score, Q[..., :64].contiguous())
    for wrong in (lambda: pg.append([2], X[:2], [1]), lambda: pg.append([2], X[:2]), lambda: pg.append([2], X[0], [1]),
                  lambda: pg.append([2], X.half(), [64]), lambda: pg.append([2], X.cpu(), [64]),
                  lambda: pg.append([2], X.view(1, 64, 128), [65]), lambda: pg.fork([0, 1], [2]),
                  lambda: pg.copy([0], [2], None, [1]), lambda: pg.copy([0], [2], [2], [1]),
                  lambda: pg.score(X), lambda: pg.score(Q.double()),
                  lambda: pg.score(Q, torch.zeros(1, 3, device="cuda")),
                  lambda: pg.score(Q, torch.zeros(2, 3, dtype=torch.int32, device="cuda")),
                  lambda: pg.score(Q, out=torch.zeros(1, 4, device="cuda")),
                  lambda: pg.read([0], out=torch.zeros(19, 128, device="cuda"))):
        with pytest.raises(ValueError):
            wrong()
    # the C entry itself: alignment, types, lists longer than the store
    L, h, one = chimera.lib(), pg._h, (ctypes.c_int64 * 1)(2)
    n1, s = (ctypes.c_int32 * 1)(1), torch.cuda.current_stream().cuda_stream
    sc = torch.full((8,), 7.0, device="cuda")
    assert L.chimera_pages_append(h, one, n1, 1, X.data_ptr() + 4, 0, 128, 128, 0, s) == bad
    assert L.chimera_pages_append(h, one, n1, 1, X.data_ptr(), 0, 128, 127, 0, s) == bad
    assert L.chimera_pages_append(h, one, n1, 1, X.data_ptr(), 1, 128, 132, 0, s) == bad
    assert L.chimera_pages_append(h, one, n1, 1, X.data_ptr(), 2, 128, 128, 0, s) == bad
    assert L.chimera_pages_append(h, one, n1, 1, None, 0, 128, 128, 0, s) == bad
    assert L.chimera_pages_append(h, one, n1, -1, X.data_ptr(), 0, 128, 128, 0, s) == bad
    assert L.chimera_pages_score(h, Q.data_ptr(), 0, 1, 32, 128, None, 6, 0, sc.data_ptr(), s) == bad
    assert L.chimera_pages_score(h, Q.data_ptr() + 4, 0, 1, 32, 128, None, 5, 0, sc.data_ptr(), s) == bad
    assert L.chimera_pages_score(h, Q.data_ptr(), 0, 1, 0, 128, None, 5, 0, sc.data_ptr(), s) == bad
    assert L.chimera_pages_score(h, Q.data_ptr(), 0, 1, 32, 128, sc.data_ptr(), 5, 4, sc.data_ptr(), s) == bad
    assert L.chimera_pages_score(h, Q.data_ptr(), 0, 1, 32, 128, None, 2**28 + 1, 0, sc.data_ptr(),
                                 s) == chimera.E_UNSUPPORTED
    assert L.chimera_pages_read(h, one, 1, X.data_ptr() + 8, 64, 0, s) == bad
    two = (ctypes.c_int64 * 2)(0, 1)
    held = torch.full((53, 128), 7.0, device="cuda")
    for rows in (52, 0, -1):  # as after another thread's append between the lengths and the read
        assert L.chimera_pages_read(h, two, 2, held.data_ptr(), rows, 0, s) == bad
    torch.cuda.synchronize()
    assert torch.all(held == 7.0)
    torch.cuda.synchronize()
    assert torch.all(sc == 7.0) and pg.info() == info
    same(pg.read([0, 1, 2, 3, 4]), np.concatenate(docs))


def test_calls_of_nothing():
    pg = Pages(1, 1, 1)
    X = torch.empty(0, 128, device="cuda")
    pg.append([], X, [])
    pg.append([0], X, [0])
    pg.append([0], torch.empty(1, 0, 128, device="cuda"))
    pg.fork([], [])
    pg.copy([], [])
    pg.copy([0], [0])
    pg.drop([])
    pg.drop([0])
    assert pg.read([]).shape == (0, 128) and pg.read([0]).shape == (0, 128)
    assert pg.score(torch.empty(0, 32, 128, device="cuda")).shape == (0, 1)
    Q = torch.ones(2, 1, 128, device="cuda")
    assert pg.score(Q, torch.empty(2, 0, dtype=torch.int32, device="cuda")).shape == (2, 0)
    assert torch.isneginf(pg.score(Q)).all()
    with pytest.raises(ChimeraError) as e:
        Pages(1, 1, 1, device=99)
    assert e.value.code == chimera.E_INVAL
