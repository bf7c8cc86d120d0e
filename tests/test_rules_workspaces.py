"""Workspaces of the attention with rules that are asked for with bounds of more than one launch takes.  No GPU."""
import shutil

import pytest

import launch_spy as S
import rules_util as U
from paper_2506_17286_amd import binding as B

MANY = [1, 100, 5000, 1 << 20, 1 << 24, 1 << 26, 1 << 27, 1 << 28, 1 << 29, 1 << 30, (1 << 31) - 300, (1 << 31) - 1, 1 << 40, (1 << 63) - 1]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", sorted(U.SHAPES) + ["k16x64l256"])
def test_a_larger_bound_never_asks_for_less(name, dtype):
    cfg = U.config(name, dtype)
    for batch in (1, 30, 3000, 65535):
        sizes = [B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFILL_MASKED, batch, t, 1 << 30) for t in MANY]
        assert sizes == sorted(sizes), batch
    for t in MANY:
        sizes = [B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFILL_MASKED, b, t, 1 << 30) for b in (1, 2, 30, 300, 3000, 65535)]
        assert sizes == sorted(sizes), t
        assert sizes[0] < 1 << 30      # (what a bound of any size costs at most)


def test_many_maps_and_sequences():
    """512 maps on one key: 65535 sequences of them are more rows than a launch takes, 32767 are not."""
    for dtype in ("bf16", "f32"):
        cfg = B.make_config(d_model=256, n_heads=512, n_qgroups=512, n_kgroups=1, n_cgroups=1, head_dim=64, latent_dim=128, dtype=dtype)
        sizes = [B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFIX_DECODE, b, 1000, 1000) for b in (1, 64, 3000, 32767, 32768, 65535)]
        assert sizes == sorted(sizes)


@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not found")
def test_they_do_for_the_calls_that_a_launch_takes():
    out = S.run("""
import rules_util as U
for name, sh in U.SHAPES.items():
    for dt in ("bf16", "f32"):
        cfg = B.make_config(dtype=dt, **sh)
        q, k, c = sh["n_qgroups"] * sh["head_dim"], sh["n_kgroups"] * sh["head_dim"], sh["n_cgroups"] * sh["latent_dim"]
        for most in (1 << 30, (1 << 31) - 1):
            n = B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFILL_MASKED, 65535, most, most)
            for batch, total in ((1, 1), (1, 3000), (7, 20000), (65535, 1 << 20), (1, 1 << 26), (300, 1 << 28), (1, 1 << 30)):
                rc = B.load().gta_prefill_masked_attention(R(cfg), FAKE, q, FAKE, k, FAKE, c, FAKE, batch, total, total, None, FAKE, FAKE, n, None)
                out.append([rc, [name, dt, most, batch, total]])
for dt in ("bf16", "f32"):
    cfg = B.make_config(d_model=256, n_heads=512, n_qgroups=512, n_kgroups=1, n_cgroups=1, head_dim=64, latent_dim=128, dtype=dt)
    n = B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFIX_DECODE, 65535, 1000, 1024)
    caches = [B.gta_cache(FAKE, FAKE, FAKE, FAKE, 65535, r, None, 0, 0, 0) for r in (1000, 1024)]
    for batch in (1, 2, 64, 65, 3000, 32767):
        rc = B.load().gta_prefix_decode_attention(R(cfg), FAKE, R(caches[0]), 0, R(caches[1]), None, batch, None, FAKE, FAKE, n, None)
        out.append([rc, [dt, batch]])
events()
""")
    assert out and all(rc == 0 for rc, _ in out), [case for rc, case in out if rc][:20]
