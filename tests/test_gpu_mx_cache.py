"""Rows quantised into 8-bit caches and read back, against the definition: every code and scale byte, nothing else touched."""
import numpy as np
import pytest
import torch

from paper_2506_17286_amd import binding as B

import mx_util as M

pytestmark = pytest.mark.gpu


def append(cache, sh, dtype, x_k, x_c, cu, max_new=None, slots=None, fused=0, offset=0):
    """x_k, x_c float64 rows (rounded to dtype here); returns what was rounded."""
    dt, total = M.DT[dtype], x_k.shape[0]
    cfg = B.make_config(dtype=dtype, **sh)
    kw, cw = x_k.shape[1], x_c.shape[1]
    buf = torch.zeros(offset + max(total, 1) * (kw + cw + fused), dtype=dt, device="cuda")[offset:].view(-1, kw + cw + fused)
    buf[:total, :kw + cw] = torch.from_numpy(np.concatenate([x_k, x_c], axis=1)).to("cuda", dt)
    k, c = buf[:, :kw], buf[:, kw:kw + cw]
    if not (fused or offset):
        k, c = k.contiguous(), c.contiguous()
    sl = None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda")
    n = max_new if max_new is not None else int(np.diff(cu).max())
    B.gta_mx_cache_append(cfg, cache.struct, sl, k, k.stride(0), c, c.stride(0), torch.tensor(cu, dtype=torch.int32, device="cuda"),
                          len(cu) - 1, n)
    torch.cuda.synchronize()
    return k[:total].double().cpu().numpy(), c[:total].double().cpu().numpy()


def expect(host, cache, slot, first, xk, xc):
    """host: the four arrays before; writes what the rows should have become"""
    at = cache.rows(slot, first, first + xk.shape[0])
    for codes, scale, x in ((host[0], host[2], xk), (host[1], host[3], xc)):
        q, s = M.quantise(x)
        codes[at], scale[at] = q, s
    return host


def same(cache, want_values, touched):
    """want_values: [k codes as numbers, c codes as numbers, ks, cs]"""
    got = cache.host()
    for i in (0, 1):
        np.testing.assert_array_equal(M.E4M3[got[i]], want_values[i])
        np.testing.assert_array_equal(got[i + 2], want_values[i + 2])
    for i in range(4):                                     # and untouched bytes are as they were, bit for bit
        keep = np.ones(got[i].shape[0], bool)
        keep[touched] = False
        assert (got[i][keep] == (0x7f, 0xff, 227, 227)[i]).all()


def numbers(cache):
    h = cache.host()
    return [M.E4M3[h[0]], M.E4M3[h[1]], h[2].copy(), h[3].copy()]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, 16, 64, 24, 1])
@pytest.mark.parametrize("name", ["1b", "paper", "odd", "tiny", "c2"])
def test_append_twice_then_read(name, page, dtype):
    sh = M.SHAPES[name]
    lens, more = [0, 1, 15, 16, 17, 100, 33], [3, 0, 1, 1, 31, 20, 1]
    cache = M.MxCache(sh, len(lens) + 2, 192, page, seed=1)
    slots = [4, 0, 8, 2, 7, 1, 5]
    rng = np.random.default_rng(2)
    want, touched, have = numbers(cache), [], {s: 0 for s in slots}
    for ns, fused, offset in ((lens, 0, 0), (more, 24, 0 if dtype == "f32" else 3)):
        cu = np.concatenate([[0], np.cumsum(ns)])
        xk, xc = (rng.standard_normal((cu[-1], w)) * np.exp2(rng.uniform(-20, 20, (cu[-1], 1))) for w in (cache.kw, cache.cw))
        xk, xc = append(cache, sh, dtype, xk, xc, cu, slots=slots, fused=fused, offset=offset)
        for b, s in enumerate(slots):
            expect(want, cache, s, have[s], xk[cu[b]:cu[b + 1]], xc[cu[b]:cu[b + 1]])
            touched.append(cache.rows(s, have[s], have[s] + ns[b]))
            have[s] += ns[b]
        same(cache, want, np.concatenate(touched))
        got = cache.seq_lens.cpu().numpy()
        assert all(got[s] == n for s, n in have.items()) and got[3] == got[6] == 0
    assert not cache.status.any()

    # read everything back, and a middle piece, with rows of other sequences around them
    cfg, dt = B.make_config(dtype=dtype, **sh), M.DT[dtype]
    host = cache.host()
    for first, ns in (([0] * 7, [have[s] for s in slots]), ([2, 0, 5, 16, 40, 90, 30], [1, 1, 40, 1, 8, 60, 0])):
        cu = np.concatenate([[0], np.cumsum(ns)])
        k, c = (torch.full((cu[-1] + 2, w), 9.0, dtype=dt, device="cuda") for w in (cache.kw, cache.cw))
        B.gta_mx_cache_read(cfg, cache.struct, torch.tensor(slots, dtype=torch.int32, device="cuda"),
                            None if not any(first) else torch.tensor(first, dtype=torch.int32, device="cuda"),
                            torch.tensor(cu, dtype=torch.int32, device="cuda"), 7, max(ns), k, c)
        for out, i in ((k, 0), (c, 1)):
            got = out.double().cpu().numpy()
            ref = np.zeros((cu[-1], got.shape[1]))
            for b, s in enumerate(slots):
                n = max(0, min(ns[b], have[s] - first[b]))   # rows behind the sequence's end read as zeros
                at = cache.rows(s, first[b], first[b] + n)
                ref[cu[b]:cu[b] + n] = M.values(host[i][at], host[i + 2][at])
            np.testing.assert_array_equal(got[:-2], ref)
            assert (got[-2:] == 9.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_16_bit_number_and_the_ends_of_the_range(dtype):
    """All bf16 patterns (NaN and infinities among them) in blocks of neighbours and in mixed blocks, and for fp32 random bit
    patterns and the borders of the exponent rule."""
    sh = M.shape(1, 1, 1, 64, 64)
    bits = np.arange(65536, dtype=np.uint32)
    near = (bits << 16).view(np.float32).astype(float).reshape(-1, 64)
    mixed = np.random.default_rng(0).permutation(near.reshape(-1)).reshape(-1, 64)
    rows = [near, mixed]
    e = np.arange(-125, 128)
    edge = np.zeros((len(e) * 3, 64))
    for i, f in enumerate((1.75, np.nextafter(np.float32(1.75), np.float32(2)), np.nextafter(np.float32(1.75), np.float32(1)))):
        edge[i * len(e):(i + 1) * len(e), 0] = float(f) * 2.0 ** e
        edge[i * len(e):(i + 1) * len(e), 5] = -float(f) * 2.0 ** (e - 9.0)
    rows.append(edge)
    ties = np.outer(2.0 ** np.arange(-16, 9), (1 + (2 * np.arange(64) + 1) / 128))   # half way between codes
    ties[:, 0] = ties[:, 32] = 448.0
    rows.append(ties)
    if dtype == "f32":
        r = np.random.default_rng(1).integers(0, 1 << 32, (2048, 64), dtype=np.uint64).astype(np.uint32).view(np.float32)
        rows.append(r.astype(float))
    with np.errstate(invalid="ignore", over="ignore"):
        x = np.concatenate(rows)
        cache = M.MxCache(sh, 1, x.shape[0])
        xk, xc = append(cache, sh, dtype, x, x[::-1].copy(), [0, x.shape[0]])
        want = numbers(cache)
        expect(want, cache, 0, 0, xk, xc)
    same(cache, want, np.arange(x.shape[0]))
    assert cache.host()[2].min() >= 10 and cache.host()[2].max() <= 246
    # what was stored reads back exactly in either precision
    for d2 in ("bf16", "f32"):
        k, c = (torch.empty((x.shape[0], 64), dtype=M.DT[d2], device="cuda") for _ in range(2))
        B.gta_mx_cache_read(B.make_config(dtype=d2, **sh), cache.struct, None, None, torch.tensor([0, x.shape[0]], dtype=torch.int32, device="cuda"),
                            1, x.shape[0], k, c)
        h = cache.host()
        np.testing.assert_array_equal(k.double().cpu().numpy(), M.values(h[0], h[2]))
        np.testing.assert_array_equal(c.double().cpu().numpy(), M.values(h[1], h[3]))


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("longest", [3, 200])              # one launch, or two
def test_sequences_that_do_not_fit_store_nothing(longest, page):
    sh = M.SHAPES["1b"]
    cache = M.MxCache(sh, 6, 256, page, missing=[(3, 8)] if page else ())
    start = [256 - longest + 1, 0, 256 - longest, 128 - 2, 10, 4]
    cache.seq_lens.copy_(torch.tensor(start, dtype=torch.int32))
    ns = [longest, longest, longest, longest, longest + 1, 0]   # full, fits, fits exactly, lacks a page, over the bound, nothing
    cu = np.concatenate([[0], np.cumsum(ns)])
    rng = np.random.default_rng(0)
    want = numbers(cache)
    xk, xc = append(cache, sh, "bf16", rng.standard_normal((cu[-1], 512)), rng.standard_normal((cu[-1], 512)), cu, max_new=longest)
    fits = [1, 2] + ([] if page else [3] if 126 + longest <= 256 else [])
    for b in fits:
        expect(want, cache, b, start[b], xk[cu[b]:cu[b + 1]], xc[cu[b]:cu[b + 1]])
    same(cache, want, np.concatenate([cache.rows(b, start[b], start[b] + ns[b]) for b in fits]))
    lens = [n + (ns[b] if b in fits else 0) for b, n in enumerate(start)]
    assert cache.seq_lens.cpu().tolist() == lens
    flags = [B.GTA_ERR_CACHE_FULL, 0, 0, 0 if 3 in fits else B.GTA_ERR_CACHE_FULL, B.GTA_ERR_SHAPE, 0]
    assert cache.status.cpu().tolist() == flags


def test_slots_out_of_range_and_lengths_out_of_range():
    sh = M.SHAPES["paper"]
    cache = M.MxCache(sh, 3, 32)
    cache.seq_lens.copy_(torch.tensor([-2, 0, 40], dtype=torch.int32))
    want = numbers(cache)
    x = np.random.default_rng(0).standard_normal((5, 192))
    xk, xc = append(cache, sh, "f32", x[:, :64], x[:, 64:], [0, 1, 2, 3, 4, 5], slots=[7, 1, -1, 0, 2])
    expect(want, cache, 1, 0, xk[1:2], xc[1:2])
    same(cache, want, cache.rows(1, 0, 1))
    assert cache.seq_lens.cpu().tolist() == [-2, 1, 40]
    assert cache.status.cpu().tolist() == [B.GTA_ERR_CACHE_FULL, 0, B.GTA_ERR_CACHE_FULL]
    # reads: slots and lengths out of range, first rows below zero, missing rows are zeros; a bound that is too small
    k, c = (torch.full((12, w), 3.0, device="cuda") for w in (64, 128))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")   # noqa: E731
    cache.status.zero_()
    cache.seq_lens.copy_(i32([-2, 1, 1]))
    B.gta_mx_cache_read(B.make_config(dtype="f32", **sh), cache.struct, i32([7, 1, -1, 0, 1, 2]), i32([0, 0, 0, 0, -1, 0]), i32([0, 1, 3, 4, 5, 7, 10]),
                        6, 2, k, c)
    h = cache.host()
    ref = np.zeros((12, 64))
    ref[[1, 6]] = M.values(h[0], h[2])[32]
    ref[7:] = 3.0                                          # skipped: more rows than the bound; then rows behind the last
    np.testing.assert_array_equal(k.double().cpu().numpy(), ref)
    assert cache.status.cpu().tolist() == [0, 0, B.GTA_ERR_SHAPE]


def test_rows_behind_4_gib():
    """Pages whose byte offset passes 32 bits."""
    sh = M.SHAPES["1b"]
    pages, page = 34000, 256
    cache = M.MxCache(sh, 1, 512, 256)
    k, c = (torch.zeros((pages, page, 512), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, cs = (torch.zeros((pages, page, 16), dtype=torch.uint8, device="cuda") for _ in range(2))
    table = torch.tensor([[pages - 1, 3]], dtype=torch.int32, device="cuda")
    far = B.make_paged_mx_cache(k, c, ks, cs, cache.seq_lens, cache.status, table)
    x = torch.randn((300, 1024), generator=torch.Generator().manual_seed(0)).to("cuda", torch.bfloat16)
    cfg = B.make_config(dtype="bf16", **sh)
    cu = torch.tensor([0, 300], dtype=torch.int32, device="cuda")
    B.gta_mx_cache_append(cfg, far, None, x, 1024, x[:, 512:], 1024, cu, 1, 300)
    ko, co = (torch.empty((300, 512), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.gta_mx_cache_read(cfg, far, None, None, cu, 1, 300, ko, co)
    for out, src, codes in ((ko, x[:, :512], k), (co, x[:, 512:], c)):
        q, s = M.quantise(src.double().cpu().numpy())
        np.testing.assert_array_equal(out.double().cpu().numpy(), q * np.repeat(2.0 ** (s.astype(float) - 127), 32, axis=1))
        assert codes[pages - 1].any() and codes[3].any() and not codes[pages - 2].any() and not codes[0].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bounds_far_above_the_rows_there_are(dtype):
    """max_new and max_rows of 2^24 and more rows of 2048 elements: launches whose last workgroups begin 2^31 words and more behind
    the sequence's end, in a slot of 2^25 rows of which two pages are there."""
    sh = M.SHAPES["wide"]
    cache = M.MxCache(sh, 1, 2048, 1024)
    table = torch.full((1, 1 << 15), -1, dtype=torch.int32, device="cuda")
    table[:, :2] = cache.table
    cache.struct = B.make_paged_mx_cache(cache.k, cache.c, cache.ks, cache.cs, cache.seq_lens, cache.status, table)
    cache.seq_lens.fill_(1020)
    rng = np.random.default_rng(3)
    want = numbers(cache)
    xk, xc = append(cache, sh, dtype, rng.standard_normal((9, cache.kw)), rng.standard_normal((9, cache.cw)), [0, 9], max_new=(1 << 25) - 1)
    expect(want, cache, 0, 1020, xk, xc)
    same(cache, want, cache.rows(0, 1020, 1029))
    assert cache.seq_lens.tolist() == [1029] and cache.status.tolist() == [0]
    host = cache.host()
    cfg, dt, at = B.make_config(dtype=dtype, **sh), M.DT[dtype], cache.rows(0, 1021, 1029)
    k, c = (torch.full((12, w), 9.0, dtype=dt, device="cuda") for w in (cache.kw, cache.cw))
    B.gta_mx_cache_read(cfg, cache.struct, None, torch.tensor([1021], dtype=torch.int32, device="cuda"),
                        torch.tensor([0, 10], dtype=torch.int32, device="cuda"), 1, (1 << 24) + 16, k, c)
    for out, i in ((k, 0), (c, 1)):
        got = out.double().cpu().numpy()
        np.testing.assert_array_equal(got[:8], M.values(host[i][at], host[i + 2][at]))
        assert (got[8:10] == 0).all() and (got[10:] == 9.0).all()
