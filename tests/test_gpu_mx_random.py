"""Layers, batches, pages and lengths drawn at random: rows are appended in two calls, read back and attended over, each step against
its definition in float64."""
import numpy as np
import pytest
import torch

from paper_2506_17286_amd import binding as B

import mx_util as M
import test_gpu_mx_decode as D
import test_gpu_mx_cache as C

pytestmark = pytest.mark.gpu


def draw(rng):
    """A layer of at most 40 maps and rows of at most 6144 elements."""
    while True:
        nq = int(rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 15, 16, 18, 20, 24, 28, 32, 40]))
        nk, nc = (int(rng.choice([n for n in range(1, nq + 1) if nq % n == 0])) for _ in range(2))
        dh = 32 * int(rng.choice([1, 2, 2, 3, 4, 4, 5, 6, 8, 12, 16, 17]))
        dl = 32 * int(rng.integers(dh // 32, 49))
        if rng.random() < 0.4:
            dl = max(dh, int(rng.choice([64, 128, 256, 512, 1024])))
            dl = dl if dl % 32 == 0 else dh
        if nk * dh + nc * dl <= 6144:
            return M.shape(nq, nk, nc, dh, dl)


@pytest.mark.parametrize("seed", range(60))
def test_append_read_attend(seed):
    rng = np.random.default_rng(seed)
    sh, dtype = draw(rng), ("bf16", "f32")[seed % 2]
    page = int(rng.choice([0, 0, 1, 8, 16, 24, 32, 64, 256]))
    slots = int(rng.integers(1, 7))
    most = int(rng.choice([40, 300, 900]))
    max_seq = (most + 80 + (page or 1) - 1) // (page or 1) * (page or 1)
    cache = M.MxCache(sh, slots, max_seq, page, seed=seed)
    kw, cw = cache.kw, cache.cw
    order = list(rng.permutation(slots))
    want, touched, have = C.numbers(cache), [], [0] * slots
    for top in (most, 40):
        ns = [int(n) for n in rng.integers(0, top + 1, slots)]
        cu = np.concatenate([[0], np.cumsum(ns)])
        xk, xc = (rng.standard_normal((cu[-1], w)) * np.exp2(rng.uniform(-3, 3, (cu[-1], 1))) for w in (kw, cw))
        xk, xc = C.append(cache, sh, dtype, xk, xc, cu, slots=order, max_new=max(max(ns), 1) + int(rng.integers(0, 3)), fused=int(rng.choice([0, 8, 5])))
        for b, s in enumerate(order):
            C.expect(want, cache, s, have[s], xk[cu[b]:cu[b + 1]], xc[cu[b]:cu[b + 1]])
            touched.append(cache.rows(s, have[s], have[s] + ns[b]))
            have[s] += ns[b]
        C.same(cache, want, np.concatenate(touched))
    assert cache.seq_lens.cpu().tolist() == have and not cache.status.any()

    cfg, dt = B.make_config(dtype=dtype, **sh), M.DT[dtype]
    first = [int(rng.integers(0, have[s] + 1)) for s in order]
    ns = [int(rng.integers(0, 60)) for _ in order]
    cu = np.concatenate([[0], np.cumsum(ns)])
    k, c = (torch.full((cu[-1] + 1, w), 9.0, dtype=dt, device="cuda") for w in (kw, cw))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")   # noqa: E731
    B.gta_mx_cache_read(cfg, cache.struct, i32(order), i32(first), i32(cu), slots, 60, k, c)
    host = cache.host()
    for out, i in ((k, 0), (c, 1)):
        got, ref = out.double().cpu().numpy(), np.zeros((cu[-1] + 1, out.shape[1]))
        ref[-1] = 9.0
        for b, s in enumerate(order):
            n = max(0, min(ns[b], have[s] - first[b]))
            at = cache.rows(s, first[b], first[b] + n)
            ref[cu[b]:cu[b] + n] = M.values(host[i][at], host[i + 2][at])
        np.testing.assert_array_equal(got, ref)

    q = D.queries(sh, dtype, slots, seed)
    sl = i32(order)
    for splits in (0, int(rng.integers(1, 9))):
        D.check(D.attend(cache, sh, dtype, q, slots, sl, splits), cache, sh, dtype, q, order, have)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["1b", "paper", "wide", "mha", "q17", "h544"])
def test_workspaces_of_any_size_are_not_left(name, dtype):
    """Sizes from one that is refused to more than the call needs, in the middle of a larger buffer of which the rest stays as it was."""
    sh, rng = M.SHAPES[name], np.random.default_rng(31)
    lens = [900, 5, 333, 0, 64]
    cache = M.MxCache(sh, 5, 960, 16).fill(lens, rng)
    q, cfg = D.queries(sh, dtype, 5), B.make_config(dtype=dtype, **sh)
    full, one = (B.gta_workspace_bytes(cfg, B.GTA_MODE_MX_DECODE, 5, 0, 960, s) for s in (0, 1))
    refused = 0
    for size in [16, 256, one, full, full + 4096] + [int(v) // 16 * 16 for v in rng.integers(256, full, 12)]:
        big = torch.full((size + 8192,), 0xa5, dtype=torch.uint8, device="cuda")
        out = torch.full((6, sh["n_qgroups"] * sh["latent_dim"]), 5.0, dtype=M.DT[dtype], device="cuda")
        rc = B.gta_mx_decode_attention(cfg, q, cache.struct, None, 5, 0, out, big[4096:4096 + size], check=False)
        torch.cuda.synchronize()
        assert (big[:4096] == 0xa5).all() and (big[4096 + size:] == 0xa5).all() and (out[5] == 5.0).all()
        if rc == B.GTA_ERR_WORKSPACE:
            assert size < one and (out == 5.0).all() and (big == 0xa5).all()
            refused += 1
        else:
            assert rc == B.GTA_OK
            D.check(out[:5].double().cpu().numpy(), cache, sh, dtype, q, range(5), lens)
    assert refused
