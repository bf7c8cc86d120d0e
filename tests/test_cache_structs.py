"""Caches that are made without one of their arrays: the call that gets one says so.  No GPU."""
import ctypes

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
