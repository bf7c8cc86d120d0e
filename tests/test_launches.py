"""What the 8-bit cache's and the norm's calls launch, looked at without a GPU (tests/launch_spy.py)."""
import shutil

import pytest

import launch_spy as S

pytestmark = pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not found")


def test_norms_of_more_rows_than_a_launch_has_threads():
    """A launch has fewer than 2^32 threads along x: more rows than that gives the vector kernel go to the one whose workgroups go on."""
    out = S.run("""
for dt in ("bf16", "f32"):
    for nq, nk, dh in ((1, 1, 256), (1, 1, 128), (1, 1, 32), (4, 4, 256), (6, 3, 64), (1, 1, 96)):
        cfg = B.make_config(d_model=256, n_heads=nq, n_qgroups=nq, n_kgroups=nk, n_cgroups=1, head_dim=dh, latent_dim=dh, dtype=dt)
        for n in (1, 5000, 1 << 20, 1 << 27, 1 << 28, (1 << 28) + 1, (1 << 31) // (nq + nk), (1 << 31) // (nq + nk) + 1):
            rc = B.load().gta_qk_norm_rope(R(cfg), FAKE, nq * dh, FAKE, nk * dh, None, None, 1e-6, None, n, FAKE, FAKE, None)
            out.append([rc, n * (nq + nk), events()])
""")
    assert len(out) == 96
    for rc, heads, text in out:
        ev = S.parse(text)
        if heads > 1 << 31:
            assert rc == -5 and not ev                      # GTA_ERR_UNSUPPORTED
        else:
            assert rc == 0 and len(ev) == 1 and ev[0].grid[0] * ev[0].threads < 1 << 32


def test_lds_is_asked_for_before_every_launch_that_needs_it():
    """Calls of one kernel after each other that take more and more dynamic LDS: above 64 KiB the limit has to have been raised to what
    the launch takes, by this call or one before, and not by every call."""
    out = S.run("""
import mx_util as M
shapes = [M.SHAPES["h32"], M.SHAPES["q17"]]               # blocks of 10 maps, of 16
shapes += [M.shape(m, 1, 1, 64, 256) for m in (1, 11, 16, 12)] + [M.shape(m, 1, 1, 128, 1024) for m in (2, 9, 16, 16)]
shapes += [M.shape(m, m, 1, 64, 1024) for m in (1, 2, 4, 8, 16)] + list(M.SHAPES.values())
for sh in shapes:
    for dt in ("bf16", "f32"):
        for batch in (1, 1025):
            cfg = B.make_config(dtype=dt, **sh)
            cache = B.gta_mx_cache(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, batch, 4096, None, 0, 0, 0)
            rc = B.load().gta_mx_decode_attention(R(cfg), FAKE, R(cache), None, batch, 0, FAKE, FAKE, 1 << 40, None)
            out.append([rc, events()])
""")
    limit, raised = {}, 0
    for rc, text in out:
        assert rc == 0
        for ev in S.parse(text):
            if isinstance(ev, S.Attr):
                assert ev.lds > limit.get(ev.kernel, 0)
                limit[ev.kernel], raised = ev.lds, raised + 1
            else:
                assert ev.lds <= max(64 << 10, limit.get(ev.kernel, 0)) and ev.lds <= 160 << 10, ev.kernel
    assert raised


def test_every_attention_kernel_is_run_by_some_layer_of_the_tests():
    """The kernels that the library has are the ones that the tests' layers take, in both types, in batches that are cut and that are not."""
    registered, taken = S.run("""
import mx_util as M, mx_layers
taken = ""
for sh in {**M.SHAPES, **mx_layers.WIDTHS}.values():
    for dt in ("bf16", "f32"):
        for batch in (8, 1026):
            cfg = B.make_config(dtype=dt, **sh)
            cache = B.gta_mx_cache(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, batch, 384, None, 0, 0, 0)
            assert B.load().gta_mx_decode_attention(R(cfg), FAKE, R(cache), None, batch, 0, FAKE, FAKE, 1 << 40, None) == 0
            taken += events()
spy.spy_names.restype = ctypes.c_char_p
out += [spy.spy_names().decode().split(), taken]
""")
    registered = {S.attention_kernel(n) for n in registered} - {None}
    taken = {S.attention_kernel(e.kernel) for e in S.parse(taken)} - {None}
    assert len(registered) == 88 and taken == registered, sorted(registered - taken)


def test_appends_of_few_rows_are_one_launch():
    """Up to 2048 words of 16 elements a sequence: one workgroup each, which sets the length; above, a second launch does."""
    out = S.run("""
import mx_util as M
for name in ("paper", "1b", "wide"):
    sh = M.SHAPES[name]
    width = sh["n_kgroups"] * sh["head_dim"] + sh["n_cgroups"] * sh["latent_dim"]
    for dt in ("bf16", "f32"):
        for rows in (0, 1, 16, 32, 2048 * 16 // width, 2048 * 16 // width + 1, 64 * 1024 // width, 4000):
            cfg = B.make_config(dtype=dt, **sh)
            cache = B.gta_mx_cache(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 8, 4096, None, 0, 0, 0)
            kw = sh["n_kgroups"] * sh["head_dim"]
            rc = B.load().gta_mx_cache_append(R(cfg), R(cache), None, FAKE, kw, FAKE, width - kw, FAKE, 8, rows, None)
            out.append([rc, rows * width // 16, events()])
""")
    for rc, words, text in out:
        ev = S.parse(text)
        assert rc == 0 and all(e.grid[1] == 8 for e in ev[:1])
        assert len(ev) == (1 if words <= 2048 else 2) and (words > 2048 or ev[0].grid == (1, 8, 1))


def test_reads_bounded_to_no_rows_launch_nothing():
    out = S.run("""
import mx_util as M
cfg = B.make_config(dtype="bf16", **M.SHAPES["1b"])
cache = B.gta_mx_cache(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 8, 4096, None, 0, 0, 0)
for most in (0, 1):
    rc = B.load().gta_mx_cache_read(R(cfg), R(cache), None, None, FAKE, 8, most, FAKE, FAKE, None)
    out.append([rc, len(events())])
""")
    assert out[0] == [0, 0] and out[1][0] == 0 and out[1][1] > 0
