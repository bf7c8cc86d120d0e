"""Every kernel of the attention over 8-bit rows, on layers that test_gpu_mx_decode.py has none for: own widths of 64, 128 and 256
key elements with 512 and 1024 latents, latents in slices.  On all of them, and on the layers there: block exponents over the
whole range, and that fp32 queries and weights keep their 24 bits."""
import numpy as np
import pytest
import torch

from paper_2506_17286_amd import binding as B

import mx_util as M
import test_gpu_mx_decode as D
from mx_layers import WIDTHS

pytestmark = pytest.mark.gpu

ALL = {**M.SHAPES, **WIDTHS}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("name", sorted(WIDTHS))
def test_pages_and_lengths(name, page, dtype):
    sh = WIDTHS[name]
    cache = M.MxCache(sh, len(D.LENS) + 1, 384, page, seed=3).fill(D.LENS + [7], np.random.default_rng(4))
    slots = list(np.random.default_rng(5).permutation(len(D.LENS))) + [-1, 99]
    q = D.queries(sh, dtype, len(slots))
    sl = torch.tensor(slots, dtype=torch.int32, device="cuda")
    for splits in (0, 1, 3):
        D.check(D.attend(cache, sh, dtype, q, len(slots), sl, splits), cache, sh, dtype, q, slots, D.LENS)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", sorted(WIDTHS))
def test_long_contexts(name, dtype):
    sh = WIDTHS[name]
    lens = [3000, 1, 2047]
    cache = M.MxCache(sh, 3, 3200, 64, seed=6).fill(lens, np.random.default_rng(7))
    q = D.queries(sh, dtype, 3)
    for splits in (0, 7):
        D.check(D.attend(cache, sh, dtype, q, 3, None, splits), cache, sh, dtype, q, range(3), lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", sorted(WIDTHS))
def test_batches_that_are_not_cut(name, dtype):
    sh = WIDTHS[name]
    lens = [(0, 1, 3, 2)[i % 4] for i in range(1026)]
    for i, n in ((5, 70), (500, 33), (1025, 95)):
        lens[i] = n
    cache = M.MxCache(sh, 1026, 96, 32).fill(lens, np.random.default_rng(16))
    q = D.queries(sh, dtype, 1026)
    got = D.attend(cache, sh, dtype, q, 1026)
    picked = [0, 1, 2, 3, 4, 5, 6, 499, 500, 501, 1022, 1023, 1024, 1025]
    D.check(got[picked], cache, sh, dtype, q[picked], picked, lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", sorted(WIDTHS))
def test_nan_reaches_the_maps_that_read_it(name, dtype):
    sh = WIDTHS[name]
    nq, nk, nc, dh, dl = (sh[n] for n in ("n_qgroups", "n_kgroups", "n_cgroups", "head_dim", "latent_dim"))
    cache = M.MxCache(sh, 3, 128).fill([90, 90, 90], np.random.default_rng(10))
    q = D.queries(sh, dtype, 3)
    clean = D.attend(cache, sh, dtype, q, 3).reshape(3, nq, dl)
    kg, cg = nk - 1, nc - 1
    cache.k[0, 40, kg * dh + 5] = 0x7f
    cache.c[1, 89, cg * dl + 3] = 0xff
    got = D.attend(cache, sh, dtype, q, 3).reshape(3, nq, dl)
    hit = np.zeros((3, nq, dl), bool)
    for g in range(nq):
        hit[0, g, :] |= g * nk // nq == kg
        hit[1, g, 3] |= g * nc // nq == cg
    assert np.isnan(got[hit]).all()
    np.testing.assert_array_equal(got[~hit], clean[~hit])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", sorted(WIDTHS))
@pytest.mark.parametrize("how", ["climb", "jump"])
def test_scores_that_move_far_along_the_rows(name, how, dtype):
    sh, n = WIDTHS[name], 700
    cache = M.MxCache(sh, 1, 704).fill([n], np.random.default_rng(8))
    t = np.arange(n)
    size = {"climb": t / 8, "jump": np.where(t % 97 == 50, t / 4.0, 0.1)}[how]
    store(cache, np.repeat(size[:, None], cache.kw, axis=1), None)
    x = np.abs(np.random.default_rng(9).standard_normal((1, sh["n_qgroups"] * sh["head_dim"])))
    q = torch.from_numpy(x).to("cuda", M.DT[dtype])
    for splits in (1, 5):
        D.check(D.attend(cache, sh, dtype, q, 1, None, splits), cache, sh, dtype, q, [0], [n])


def store(cache, k, c):
    """Rows 0 .. of slot 0 of a contiguous cache, quantised here (None: as they are)."""
    order = np.argsort(M.E4M3[:127])
    host = cache.host()
    for i, x in ((0, k), (1, c)):
        if x is not None:
            v, scale = M.quantise(x)
            mag = order[np.searchsorted(M.E4M3[:127][order], np.abs(v))]
            host[i][:len(x)], host[i + 2][:len(x)] = (mag + 128 * np.signbit(v)).astype(np.uint8), scale
    for t, h in zip((cache.k, cache.c, cache.ks, cache.cs), host):
        t.copy_(torch.from_numpy(h).view(t.shape))


def flushed(n, dtype):
    """Products and sums below the least normal number, 2^-126, may come out as zero: up to three parts of n terms."""
    return 3 * n * 2.0 ** -126


def held(got, cache, sh, dtype, q, n):
    host, q = cache.host(), q.double().cpu().numpy()
    at = cache.rows(0, 0, n)
    ref, mag, big = M.attention(sh, q[0], M.values(host[0][at], host[2][at]), M.values(host[1][at], host[3][at]))
    bound = M.attention_bound(dtype, sh, n, ref, mag, big) + flushed(n, dtype)
    assert np.isfinite(got).all()
    worst = (np.abs(got[0] - ref) / bound).max()
    assert worst <= 1, f"{worst:.3g} of the bound"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", sorted(ALL))
def test_block_exponents_over_the_range(name, dtype):
    """Keys with exponents from -117 to 60, far apart in neighbouring blocks and up to 20 apart from row to row, and queries that
    bring their products back to ordinary scores; latents likewise, up to 79.  A byte of another block or row, or one without its
    top bit, is off by far more than the bound."""
    sh, n = ALL[name], 300
    rng = np.random.default_rng(21)
    cache = M.MxCache(sh, 1, 320).fill([n], rng)
    rows = []
    for w, ends in ((cache.kw, (-97, 60, -50, 1, 20, -20)), (cache.cw, (-97, 79, -60, 8, 0, 60, -30, 1))):
        e = np.array(ends)[(np.arange(w // 32) + (w // 32) // len(ends)) % len(ends)]
        x = rng.standard_normal((n, w)) * np.repeat(2.0 ** (e + 8.0 - rng.integers(0, 21, (n, w // 32))), 32, axis=1)
        rows.append((x, e))
    store(cache, rows[0][0], rows[1][0])
    if cache.kw >= 64:                                      # both halves of the byte's range take part
        assert cache.ks.view(-1, cache.kw // 32)[:n].min() < 60 and cache.ks.view(-1, cache.kw // 32)[:n].max() >= 128
    nq, nk, dh = sh["n_qgroups"], sh["n_kgroups"], sh["head_dim"]
    q = rng.standard_normal((nq, dh))
    for g in range(nq):
        e = rows[0][1][g * nk // nq * dh // 32:][:dh // 32]
        q[g] *= 4 * np.repeat(2.0 ** (-8.0 - e), 32)
    q = torch.from_numpy(q.reshape(1, -1)).to("cuda", M.DT[dtype])
    for splits in (1, 4):
        held(D.attend(cache, sh, dtype, q, 1, None, splits), cache, sh, dtype, q, n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", sorted(ALL))
@pytest.mark.parametrize("how", ["level", "climb"])
def test_the_largest_latents(name, how, dtype):
    """Blocks up to the largest exponent, 119, next to ordinary ones, with one sign and with both: the result is an average and
    finite.  climb: scores that rise along the rows, so that weights are taken relative to far lower ones."""
    sh, n = ALL[name], 300
    rng = np.random.default_rng(22)
    cache = M.MxCache(sh, 1, 320).fill([n], rng)
    e = np.array((119, 0, 100, 60, 119, 90, 70, 80))[np.arange(cache.cw // 32) % 8]
    c = np.clip(rng.standard_normal((n, cache.cw)) * 150, -448, 448)
    c[:, ::2] = np.abs(c[:, ::2])
    c[:, :32] = 448.0                                       # the largest there is, in every row
    size = 0.2 * np.ones(n) if how == "level" else np.arange(n) / 8
    store(cache, np.repeat(size[:, None], cache.kw, axis=1) * (1 if how == "climb" else rng.standard_normal((n, cache.kw))),
          c * np.repeat(2.0 ** e, 32))
    x = np.abs(rng.standard_normal((1, sh["n_qgroups"] * sh["head_dim"]))) * 3 / np.sqrt(sh["head_dim"])
    q = torch.from_numpy(x).to("cuda", M.DT[dtype])
    for splits in (1, 4):
        held(D.attend(cache, sh, dtype, q, 1, None, splits), cache, sh, dtype, q, n)


@pytest.mark.parametrize("name", sorted(ALL))
def test_fp32_queries_keep_24_bits(name):
    """Keys K in one element and -K in another (K a power of two), queries 1 + a 2^-20 and 1 there, a scale of 2^20: the scores are a K, and the
    sums exact if the queries are.  With 16 bits of them all scores are 0."""
    sh = ALL[name]
    nq, nk, dh = sh["n_qgroups"], sh["n_kgroups"], sh["head_dim"]
    n = 40
    rng = np.random.default_rng(23)
    cache = M.MxCache(sh, 1, 64).fill([n], rng)
    k, q, a = np.zeros((n, nk, dh)), np.zeros((nq, dh)), rng.integers(1, 5, nq)
    K = rng.choice([0.0, 0.5, 1.0, 2.0, -1.0, -0.5], n)
    spots = [rng.permutation(dh)[:2] for _ in range(nk)]
    for h, (i, j) in enumerate(spots):
        k[:, h, i], k[:, h, j] = K, -K
    for g in range(nq):
        i, j = spots[g * nk // nq]
        q[g, i], q[g, j] = 1 + a[g] * 2.0 ** -20, 1
    store(cache, k.reshape(n, -1), None)
    qt = torch.from_numpy(q.reshape(1, -1)).float().cuda()
    host, at = cache.host(), cache.rows(0, 0, n)
    ref, mag, _ = M.attention(sh, q.reshape(-1) * 2.0 ** 20 * np.sqrt(dh), M.values(host[0][at], host[2][at]), M.values(host[1][at], host[3][at]))
    # scores of at most 8: the scale in base 2, the product and the difference to the maximum (up to 12 more) round once each, the
    # exponential by a step: (8 + 8 + 12 + 2) half steps, for a weight and for the sum of them; then sums as in attention_bound
    rel = (2 * 30 + n + 64) * 2.0 ** -24
    for splits in (1, 2):
        got = D.attend(cache, sh, "f32", qt, 1, None, splits, scale=2.0 ** 20)[0]
        worst = (np.abs(got - ref) / np.maximum(rel * mag + 2.0 ** -24 * np.abs(ref), 1e-300)).max()
        assert worst <= 1, f"{worst:.3g} of the bound"


def bf16(v):
    b = (np.asarray(v, np.float32).view(np.uint32).astype(np.uint64) + 0x7fff + ((np.asarray(v, np.float32).view(np.uint32) >> 16) & 1)) & 0xffff0000
    return b.astype(np.uint32).view(np.float32).astype(float)


@pytest.mark.parametrize("name", sorted(ALL))
def test_fp32_weights_keep_24_bits(name):
    """Three rows: a score of 0 over latents of 0, and twice a score x < 0 over the same latents c: L = 2pc / (1 + 2p), p = e^x.  x is picked
    so that p is far (50 x 2^-24 of itself at least) from every sum of two bf16 numbers that a rounding in two steps gives."""
    sh = ALL[name]
    nq, nk, nc, dh, dl = (sh[n] for n in ("n_qgroups", "n_kgroups", "n_cgroups", "head_dim", "latent_dim"))
    rng = np.random.default_rng(24)
    x = np.float32(-rng.uniform(0.05, 0.65, 200000)).astype(float)
    p = np.exp(x)
    hi = bf16(p)
    x = x[np.abs(p - hi - bf16(p - hi)) / p >= 50 * 2.0 ** -24][:nq]
    assert len(x) == nq
    p = np.exp(x)
    cache = M.MxCache(sh, 1, 32).fill([3], rng)
    k, q = np.zeros((3, nk, dh)), np.zeros((nq, dh))
    at = rng.integers(0, dh, nk)
    for h in range(nk):
        k[1:, h, at[h]] = 1.0
    for g in range(nq):
        q[g, at[g * nk // nq]] = x[g]
    c = np.zeros((3, cache.cw))
    c[1:] = np.clip(rng.standard_normal(cache.cw) * 100, -448, 448)
    store(cache, k.reshape(3, -1), c)
    qt = torch.from_numpy(q.reshape(1, -1)).float().cuda()
    host = cache.host()
    cv = M.values(host[1][1], host[3][1])
    ref = np.stack([2 * p[g] * cv[g * nc // nq * dl:][:dl] / (1 + 2 * p[g]) for g in range(nq)]).reshape(-1)
    got = D.attend(cache, sh, "f32", qt, 1, None, 1, scale=1.0)[0]
    # in units of 2^-24 of the result: score in base 2 (two roundings of less than 1, times ln 2) 1.4, the exponential 2, sums of
    # three parts of two rows (the first exact, two roundings of up to 2 each for the others) 8, of the weights 2, quotient and
    # result 2
    worst = (np.abs(got - ref) / np.maximum(16 * 2.0 ** -24 * np.abs(ref), 1e-300)).max()
    assert worst <= 1, f"{worst:.3g} of the bound"


@pytest.mark.parametrize("name", sorted(ALL))
def test_fp32_queries_on_any_16_bytes(name):
    sh = ALL[name]
    lens = [300, 17, 1]
    cache = M.MxCache(sh, 3, 320).fill(lens, np.random.default_rng(25))
    q = D.queries(sh, "f32", 3)
    moved = torch.zeros(q.numel() + 4, device="cuda")[4:].view(q.shape)
    moved.copy_(q)
    assert q.data_ptr() % 32 == 0 and moved.data_ptr() % 32 == 16
    np.testing.assert_array_equal(D.attend(cache, sh, "f32", moved, 3), D.attend(cache, sh, "f32", q, 3))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_captured_call_that_takes_more_lds_than_those_before(dtype):
    """Maps in blocks of 10, then of 16 on the same kernel: the second call asks for more LDS, here for the first time within a capture."""
    small, sh = M.shape(20, 4, 2, 32, 640), M.shape(16, 1, 1, 96, 1280)
    warm = M.MxCache(small, 2, 64).fill([40, 3], np.random.default_rng(26))
    D.attend(warm, small, dtype, D.queries(small, dtype, 2), 2)
    lens = [300, 17, 0]
    cache = M.MxCache(sh, 3, 320, 16).fill(lens, np.random.default_rng(27))
    q, cfg = D.queries(sh, dtype, 3), B.make_config(dtype=dtype, **sh)
    ws = B.alloc_workspace(B.gta_workspace_bytes(cfg, B.GTA_MODE_MX_DECODE, 3, 0, 320))
    out = torch.zeros((3, 16 * 1280), dtype=M.DT[dtype], device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        B.gta_mx_decode_attention(cfg, q, cache.struct, None, 3, 0, out, ws, stream=side)
    for _ in range(3):
        out.fill_(7.0)
        ws.view(torch.uint8).fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        got = out.double().cpu().numpy()
        np.testing.assert_array_equal(got, D.attend(cache, sh, dtype, q, 3))
        D.check(got, cache, sh, dtype, q, range(3), lens)
