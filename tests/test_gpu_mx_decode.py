"""Attention of one token over 8-bit rows against softmax in float64: groupings, lengths around every tile and page border,
empty sequences, splits, rows that must not be read, values that are not finite."""
import numpy as np
import pytest
import torch

from paper_2506_17286_amd import binding as B

import mx_util as M

pytestmark = pytest.mark.gpu

LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300]


def attend(cache, sh, dtype, q, batch, slots=None, splits=0, scale=0.0, ws_bytes=None):
    cfg = B.make_config(dtype=dtype, softmax_scale=scale, **sh)
    ws = B.alloc_workspace(B.gta_workspace_bytes(cfg, B.GTA_MODE_MX_DECODE, batch, 0, cache.max_seq, splits) if ws_bytes is None else ws_bytes)
    ws.view(torch.uint8).fill_(0xff)                       # NaN: nothing may be taken from it
    out = torch.full((batch + 1, sh["n_qgroups"] * sh["latent_dim"]), 5.0, dtype=M.DT[dtype], device="cuda")
    B.gta_mx_decode_attention(cfg, q, cache.struct, slots, batch, splits, out, ws)
    torch.cuda.synchronize()
    assert (out[batch] == 5.0).all()
    return out[:batch].double().cpu().numpy()


def queries(sh, dtype, batch, seed=0, size=1.0):
    w = sh["n_qgroups"] * sh["head_dim"]
    x = np.random.default_rng(1000 + seed).standard_normal((batch, w)) * size
    return torch.from_numpy(x).to("cuda", M.DT[dtype])


def check(got, cache, sh, dtype, q, slots, lens):
    host, q = cache.host(), q.double().cpu().numpy()
    worst = 0.0
    for b, s in enumerate(slots):
        n = lens[s] if 0 <= s < len(lens) else 0
        at = cache.rows(s, 0, n) if n else np.zeros(0, np.int64)
        ref, mag, big = M.attention(sh, q[b], M.values(host[0][at], host[2][at]), M.values(host[1][at], host[3][at]))
        bound = M.attention_bound(dtype, sh, n, ref, mag, big)
        if n == 0:
            assert (got[b] == 0).all()
            continue
        ratio = np.abs(got[b] - ref) / np.maximum(bound, 1e-300)   # (one row whose latent is 0: 0 off, 0 allowed)
        assert np.isfinite(ratio).all(), f"sequence {b} of {n} rows"
        worst = max(worst, ratio.max())
        assert ratio.max() <= 1, f"sequence {b} of {n} rows: {ratio.max():.2f} of the bound"
    return worst


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, 16, 64, 24])
@pytest.mark.parametrize("name", sorted(M.SHAPES))
def test_groupings_pages_and_lengths(name, page, dtype):
    sh = M.SHAPES[name]
    max_seq = 384
    cache = M.MxCache(sh, len(LENS) + 1, max_seq, page, seed=3).fill(LENS + [7], np.random.default_rng(4))
    slots = list(np.random.default_rng(5).permutation(len(LENS))) + [-1, 99]
    q = queries(sh, dtype, len(slots))
    sl = torch.tensor(slots, dtype=torch.int32, device="cuda")
    for splits in (0, 1, 3):
        got = attend(cache, sh, dtype, q, len(slots), sl, splits)
        check(got, cache, sh, dtype, q, slots, LENS)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name,page", [("1b", 64), ("paper", 0), ("wide", 16), ("gta4", 64), ("odd", 0), ("c4", 0), ("tiny", 16),
                                       ("q17", 64), ("h160", 0), ("mha", 64), ("h544", 0), ("1b", 40)])
def test_long_contexts_and_splits(name, page, dtype):
    sh = M.SHAPES[name]
    lens = [5000, 1, 2047, 4097]
    cache = M.MxCache(sh, 4, 5120, page, seed=6).fill(lens, np.random.default_rng(7))
    q = queries(sh, dtype, 4)
    for splits in (0, 1, 2, 7, 64, 1024):
        check(attend(cache, sh, dtype, q, 4, None, splits), cache, sh, dtype, q, range(4), lens)
    # a workspace that holds one split only
    one = B.gta_workspace_bytes(B.make_config(dtype=dtype, **sh), B.GTA_MODE_MX_DECODE, 4, 0, 5120, 1)
    check(attend(cache, sh, dtype, q, 4, None, 0, ws_bytes=one), cache, sh, dtype, q, range(4), lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["1b", "paper", "odd", "h544"])
@pytest.mark.parametrize("how", ["climb", "fall", "jump", "flat", "zero"])
def test_scores_that_move_far_along_the_rows(name, how, dtype):
    """The running maximum climbs, falls or jumps by hundreds (in units of the exponent); all keys alike; all keys zero."""
    sh = M.SHAPES[name]
    n = 700
    cache = M.MxCache(sh, 1, 704).fill([n], np.random.default_rng(8))
    at = cache.rows(0, 0, n)
    host = cache.host()
    t = np.arange(n)
    size = {"climb": t / 8, "fall": (n - t) / 8, "jump": np.where(t % 97 == 50, t / 4.0, 0.1), "flat": np.ones(n), "zero": np.zeros(n)}[how]
    codes, scale = M.quantise(np.repeat(size[:, None], cache.kw, axis=1))
    order = np.argsort(M.E4M3[:127])
    host[0][at], host[2][at] = order[np.searchsorted(M.E4M3[:127][order], codes)].astype(np.uint8), scale
    cache.k.copy_(torch.from_numpy(host[0]).view(cache.k.shape))
    cache.ks.copy_(torch.from_numpy(host[2]).view(cache.ks.shape))
    x = np.abs(np.random.default_rng(9).standard_normal((1, sh["n_qgroups"] * sh["head_dim"])))
    q = torch.from_numpy(x).to("cuda", M.DT[dtype])
    for splits in (1, 5):
        check(attend(cache, sh, dtype, q, 1, None, splits), cache, sh, dtype, q, [0], [n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["1b", "q8k4", "wide", "odd", "mha", "c2", "k5", "h32", "h160", "w672", "q40", "h544"])
def test_nan_reaches_the_maps_that_read_it(name, dtype):
    """A NaN key code: every latent of the maps of that key, no other map.  A NaN latent code: that latent of its maps."""
    sh = M.SHAPES[name]
    nq, nk, nc, dh, dl = (sh[n] for n in ("n_qgroups", "n_kgroups", "n_cgroups", "head_dim", "latent_dim"))
    lens = [90, 90, 90]
    cache = M.MxCache(sh, 3, 128).fill(lens, np.random.default_rng(10))
    q = queries(sh, dtype, 3)
    clean = attend(cache, sh, dtype, q, 3)
    kg, cg = nk - 1, nc - 1
    cache.k[0, 40, kg * dh + 5] = 0x7f
    cache.c[1, 89, cg * dl + 3] = 0xff
    for splits in (0, 4):
        got = attend(cache, sh, dtype, q, 3, None, splits).reshape(3, nq, dl)
        hit = np.zeros((3, nq, dl), bool)
        for g in range(nq):
            hit[0, g, :] |= g * nk // nq == kg
            hit[1, g, 3] |= g * nc // nq == cg
        assert np.isnan(got[hit]).all() and np.isfinite(got[~hit]).all()
        if splits == 0:
            np.testing.assert_array_equal(got[~hit], clean.reshape(3, nq, dl)[~hit])


def test_softmax_scale_and_lengths_out_of_range():
    sh = M.SHAPES["1b"]
    cache = M.MxCache(sh, 4, 64).fill([64, 64, 64, 64], np.random.default_rng(11))
    q = queries(sh, "f32", 4)
    same = attend(cache, sh, "f32", q, 4, scale=1 / np.sqrt(128))
    np.testing.assert_array_equal(same, attend(cache, sh, "f32", q, 4))
    other = attend(cache, sh, "f32", q * 2, 4, scale=0.5 / np.sqrt(128))
    np.testing.assert_array_equal(same, other)             # powers of two change no rounding
    cache.seq_lens.copy_(torch.tensor([64, 1 << 30, -5, 0], dtype=torch.int32))
    got = attend(cache, sh, "f32", q, 4)
    np.testing.assert_array_equal(got[:2], same[:2])       # a length beyond the slot's rows counts as all of them
    assert (got[2:] == 0).all()


@pytest.mark.parametrize("name", ["1b", "odd"])
def test_a_missing_page_is_read_from_page_0(name):
    sh = M.SHAPES[name]
    cache = M.MxCache(sh, 1, 96, 16, seed=2).fill([96], np.random.default_rng(12))
    q = queries(sh, "f32", 1)
    cache.table[0, 2], cache.table[0, 4] = 0, 0
    want = attend(cache, sh, "f32", q, 1)
    cache.table[0, 2], cache.table[0, 4] = -7, 1 << 30
    np.testing.assert_array_equal(attend(cache, sh, "f32", q, 1), want)


@pytest.mark.parametrize("name", ["1b", "odd"])
def test_pages_behind_4_gib(name):
    sh = M.SHAPES[name]
    small = M.MxCache(sh, 1, 512, 64, seed=1).fill([500], np.random.default_rng(13))
    pages = (5 << 30) // (64 * min(small.kw, small.cw)) + 8
    far = M.MxCache.__new__(M.MxCache)
    far.__dict__.update(small.__dict__)
    big = [torch.zeros((pages, 64, t.shape[-1]), dtype=torch.uint8, device="cuda") for t in (small.k, small.c, small.ks, small.cs)]
    n = small.k.shape[0]
    for t, s in zip(big, (small.k, small.c, small.ks, small.cs)):
        t[pages - n:] = s
    table = small.table + (pages - n)
    far.struct = B.make_paged_mx_cache(*big, small.seq_lens, small.status, table)
    q = queries(sh, "bf16", 1)
    np.testing.assert_array_equal(attend(far, sh, "bf16", q, 1), attend(small, sh, "bf16", q, 1))


@pytest.mark.parametrize("batch", [63, 64, 65, 256, 257, 700, 1024, 1025])
@pytest.mark.parametrize("name,dtype", [("paper", "f32"), ("1b", "bf16")])
def test_batches_around_the_ways_of_cutting_them(name, dtype, batch):
    """Up to 64 sequences, up to 1024, and more are cut into pieces in ways of their own; lengths from none to a few tiles, a
    few long ones between them."""
    sh = M.SHAPES[name]
    rng = np.random.default_rng(batch)
    lens = [int(n) for n in rng.choice([0, 1, 5, 31, 32, 33, 64, 130], batch)]
    lens[batch // 2] = 380
    cache = M.MxCache(sh, batch, 384, 16 if batch % 2 else 0, seed=1).fill(lens, rng)
    q = queries(sh, dtype, batch)
    for splits in (0, 1, 3):
        check(attend(cache, sh, dtype, q, batch, None, splits), cache, sh, dtype, q, range(batch), lens)


@pytest.mark.parametrize("name", ["paper", "1b", "wide", "c2"])
def test_one_long_sequence_among_many_short(name):
    sh = M.SHAPES[name]
    for batch in (40, 90):
        lens = [3 + i % 60 for i in range(batch)]
        lens[7], lens[20], lens[batch - 1] = 9000, 0, 4000
        rng = np.random.default_rng(batch)
        cache = M.MxCache(sh, batch, 9024, 64, seed=5).fill(lens, rng)
        q = queries(sh, "bf16", batch)
        check(attend(cache, sh, "bf16", q, batch), cache, sh, "bf16", q, range(batch), lens)


@pytest.mark.parametrize("name", ["paper", "1b", "wide"])
def test_same_results_from_run_to_run_and_in_any_order_of_the_batch(name):
    """No atomics: the same call gives the same bits.  Sequences that two batches cut alike do, too."""
    sh = M.SHAPES[name]
    lens = [700, 2500, 33, 0, 1290, 64, 5000, 1]
    cache = M.MxCache(sh, 8, 5120, 64, seed=3).fill(lens, np.random.default_rng(15))
    q = queries(sh, "bf16", 8)
    first = attend(cache, sh, "bf16", q, 8)
    for _ in range(3):
        np.testing.assert_array_equal(attend(cache, sh, "bf16", q, 8), first)
    order = [5, 1, 7, 0, 2, 6, 3, 4]
    sl = torch.tensor(order, dtype=torch.int32, device="cuda")
    got = attend(cache, sh, "bf16", q[torch.tensor(order, device="cuda")].contiguous(), 8, sl, 4)
    np.testing.assert_array_equal(got, attend(cache, sh, "bf16", q, 8, None, 4)[order])
    twice = torch.tensor([1, 1, 1], dtype=torch.int32, device="cuda")     # a slot more than once
    got = attend(cache, sh, "bf16", q[[1, 1, 1]].contiguous(), 3, twice, 4)
    for b in range(3):
        np.testing.assert_array_equal(got[b], attend(cache, sh, "bf16", q, 8, None, 4)[1])


@pytest.mark.parametrize("name", ["paper", "h32", "q17"])
def test_large_batches(name):
    """More sequences than fill the chip, of a row or two and of none."""
    sh = M.SHAPES[name]
    lens = [i % 5 for i in range(3000)]
    cache = M.MxCache(sh, 3000, 16).fill(lens, np.random.default_rng(14))
    q = queries(sh, "bf16", 3000)
    got = attend(cache, sh, "bf16", q, 3000)
    check(got, cache, sh, "bf16", q, range(3000), lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", sorted(M.SHAPES))
def test_batches_that_are_not_cut(name, dtype):
    """A workgroup per sequence: more than 1024 of them, of no rows to a few tiles."""
    sh = M.SHAPES[name]
    lens = [(0, 1, 3, 2)[i % 4] for i in range(1026)]
    for i, n in ((5, 70), (500, 33), (1025, 95)):
        lens[i] = n
    cache = M.MxCache(sh, 1026, 96, 32).fill(lens, np.random.default_rng(16))
    q = queries(sh, dtype, 1026)
    got = attend(cache, sh, dtype, q, 1026)
    picked = [0, 1, 2, 3, 4, 5, 6, 499, 500, 501, 1022, 1023, 1024, 1025]
    check(got[picked], cache, sh, dtype, q[picked], picked, lens)
