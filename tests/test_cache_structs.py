"""Caches of arrays that are missing or do not belong together: the call that gets one says so.  No GPU."""
import ctypes

import pytest
import torch

from paper_2506_17286_amd import binding as B

FAKE = 4096   # never dereferenced: every call below is refused first


def test_a_cache_without_latents():
    cfg = B.make_config(d_model=256, n_heads=4, n_qgroups=4, n_kgroups=4, n_cgroups=1, head_dim=64, latent_dim=128, dtype="bf16")
    k, n = torch.zeros(2, 64, 256, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    table = torch.zeros(2, 1, dtype=torch.int32)
    whole = B.make_cache(k, torch.zeros(2, 64, 128, dtype=torch.bfloat16), n, n)
    for cache in (B.make_cache(k, None, n, n), B.make_paged_cache(k, None, n, n, table)):
        assert cache.c is None and cache.k == k.data_ptr()
        assert B.load().gta_prefix_decode_attention(ctypes.byref(cfg), FAKE, ctypes.byref(whole), 0, B._rows_of(-1, cfg, cache), None, 1, None, FAKE, FAKE,
                                                    1 << 40, None) == B.GTA_ERR_NULL


def _bad(paged):
    """Arrays that do not belong together: a call would read past their end, or something else than is there."""
    lead = (10, 16) if paged else (2, 64)
    bf = dict(dtype=torch.bfloat16)
    bad = [dict(c=torch.zeros(*lead, 128)), dict(c=torch.zeros(*lead, 128, dtype=torch.float16)), dict(c=torch.zeros(lead[0] - 1, lead[1], 128, **bf)),
           dict(c=torch.zeros(lead[0], lead[1] // 2, 128, **bf)), dict(c=torch.zeros(*lead, 256, **bf)[..., ::2]),
           dict(c=torch.zeros(*lead, 256, **bf)[..., :128]), dict(k=torch.zeros(*lead, 512, **bf)[..., :256]), dict(c=torch.zeros(*lead, 128, device="meta", **bf)),
           dict(seq_lens=torch.zeros(2, dtype=torch.int64)), dict(seq_lens=torch.zeros(1, dtype=torch.int32)),
           dict(seq_lens=torch.zeros(4, dtype=torch.int32)[::2]), dict(seq_lens=torch.zeros(2, dtype=torch.int32, device="meta"))]
    if paged:
        bad += [dict(table=torch.zeros(2, 4, dtype=torch.int64)), dict(table=torch.zeros(2, 8, dtype=torch.int32)[:, ::2]),
                dict(table=torch.zeros(2, 4, dtype=torch.int32, device="meta"))]
    return bad


def test_arrays_that_do_not_belong_together():
    cfg = B.make_config(d_model=256, n_heads=4, n_qgroups=4, n_kgroups=4, n_cgroups=1, head_dim=64, latent_dim=128, dtype="bf16")
    for paged in (False, True):
        lead = (10, 16) if paged else (2, 64)
        good = dict(k=torch.zeros(*lead, 256, dtype=torch.bfloat16), c=torch.zeros(*lead, 128, dtype=torch.bfloat16),
                    seq_lens=torch.zeros(2, dtype=torch.int32), status=torch.zeros(2, dtype=torch.int32), table=torch.zeros(2, 4, dtype=torch.int32))

        def cache(**kw):
            a = dict(good, **kw)
            table = a.pop("table")
            return B.make_paged_cache(*a.values(), table) if paged else B.make_cache(*a.values())
        assert B._rows_of(-1, cfg, cache()) is not None
        for kw in _bad(paged):
            made = cache(**kw)                 # (other calls take what they took)
            with pytest.raises(ValueError):
                B._rows_of(-1, cfg, made)
