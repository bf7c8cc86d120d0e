"""Attention with rules over latents near the end of the range: the average of finite latents is finite."""
import pytest
import torch

import rules_util as R
import test_gpu_masked_attention as M
import test_gpu_prefix_decode as P

pytestmark = pytest.mark.gpu

SIGNS = ["one", "both", "few"]


def large(c, signs):
    """Latents of 1e38 to 3e38, all positive or of both signs; or such ones in a few rows and columns."""
    if c.numel() == 0:
        return
    x = c.float()
    size = (1.0 + 2.0 * x.abs().clamp(max=1.0)) * 1e38
    if signs == "both":
        size = size * x.sign()
    if signs == "few":
        keep = x.clone()
        keep[..., ::97, 3:40] = size[..., ::97, 3:40]
        size = keep
    c.copy_(size.to(c.dtype))


def lifted(q, k):
    """Scores that rise from the last key to the first, some by more than what a kernel leaves its sums' reference alone for."""
    q.copy_(q.abs())
    n = k.shape[-2]
    k.copy_((0.3 * k.float() + 0.5 * torch.linspace(1.0, 0.0, n, device="cuda")[:, None]).to(k.dtype))


@pytest.mark.parametrize("signs", SIGNS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["paper", "1b", "wide", "l192", "q6k2c3", "odd", "h96"])
def test_prompts(name, dtype, signs):
    for lift in (False, True):
        def edit(q, k, c, lo, hi):
            large(c, signs)
            if lift:
                lifted(q, k)
        M.run(name, dtype, [40, 300], "causal", edit=edit, seed=71)
        M.run(name, dtype, [150, 400], "documents", edit=edit, seed=72, longest=3000, cap=20.0)
        M.run(name, dtype, [1700], "window", edit=edit, seed=73, bias=True)


@pytest.mark.parametrize("signs", SIGNS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name,page", [("paper", 0), ("1b", 64), ("wide", 0), ("l256", 16), ("c2", 0), ("l192", 0), ("odd", 5), ("h96", 0)])
def test_prefixes(name, page, dtype, signs):
    for lift in (False, True):
        def edit(prefix, own, q):
            for t in (prefix, own):
                large(t.c, signs)
                if lift:
                    for i in range(t.k.shape[0]):
                        lifted(q, t.k[i])
                if t.pools[0] is not t.k:
                    for pool, rows in zip(t.pools, (t.k, t.c)):
                        pool[t.table.long().flatten()] = rows.view(-1, pool.shape[1], rows.shape[2])
        unit = max(page, 64) if page != 5 else 320
        P.run(name, dtype, 1500, [1, 600, 0, 17], edit=edit, seed=74, page=page, room=1280 if page == 5 else None, prefix_room=1600 if page == 5 else None)
        P.run(name, dtype, 9, [1300, 2], edit=edit, seed=75, page=page, room=1600 if page == 5 else None, prefix_room=unit, cap=30.0)
        P.run(name, dtype, 700, [20 + i for i in range(70)], edit=edit, seed=76, room=320 if page == 5 else None, prefix_room=960 if page == 5 else None, page=page)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["paper", "1b", "wide", "l192", "odd"])
@pytest.mark.parametrize("where", ["prompt", "prefix", "own"])
def test_large_latents_of_small_weights(name, dtype, where):
    """A latent of 1e38 with a weight of e^-78 = 2^-112.5 (and its neighbour of 1e37) counts for thousands of others."""
    dh = R.SHAPES[name]["head_dim"]

    def keys(k, c, row):
        k[:, :] = 0.0
        k[row, ::dh] = -78.0 * dh ** 0.5      # times a query of 1, over the root of the head: -78
        c[row] = 1e38
        c[row, 1::2] = -1e37

    def queries(q):
        q[:, :] = 0.0
        q[:, ::dh] = 1.0
    if where == "prompt":
        def edit(q, k, c, lo, hi):
            queries(q)
            keys(k, c, 500)
        for longest in (None, 5000):
            M.run(name, dtype, [1200], "whole", edit=edit, seed=77, longest=longest)
    else:
        def edit(prefix, own, q):
            queries(q)
            for t in (prefix, own):
                for i, n in enumerate(t.lens):
                    t.k[i, :n] = 0.0
            t = prefix if where == "prefix" else own
            for i, n in enumerate(t.lens):
                if n > 60:
                    keys(t.k[i, :n], t.c[i, :n], 50)
        P.run(name, dtype, 1000, [3000, 70, 5], edit=edit, seed=78)
