"""What the calls of the rotation and of the attention with rules launch, looked at without a GPU (tests/launch_spy.py)."""
import shutil

import pytest

import launch_spy as S

pytestmark = pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not found")

SETUP = """
import rules_util as U
def cfgs():
    for name, sh in {**U.SHAPES, **U.ROWS}.items():
        for dt in ("bf16", "f32"):
            yield name, dt, sh, B.make_config(dtype=dt, **sh)
def widths(sh):
    return sh["n_qgroups"] * sh["head_dim"], sh["n_kgroups"] * sh["head_dim"], sh["n_cgroups"] * sh["latent_dim"]
"""


def _fits(ev):
    return 1 <= ev.grid[0] and ev.grid[0] * ev.threads < 1 << 32 and ev.grid[1] <= 65535 and ev.grid[2] <= 65535 and ev.lds <= 160 << 10


def _check(out):
    limit = {}
    for rc, text in out:
        assert rc in (0, -5)
        events = S.parse(text)
        assert (rc == 0) == bool(events)
        for ev in events:
            if isinstance(ev, S.Attr):
                assert ev.lds > limit.get(ev.kernel, 0)
                limit[ev.kernel] = ev.lds
            else:
                assert _fits(ev), (ev, rc)
                assert ev.lds <= max(64 << 10, limit.get(ev.kernel, 0)), ev.kernel
    return limit


def test_masked_attention():
    """Launches that fit, LDS asked for before it is used, for every layer, few and very many tokens, with and without rules."""
    out = S.run(SETUP + """
for name, dt, sh, cfg in cfgs():
    q, k, c = widths(sh)
    for batch, total, longest in ((1, 1, 1), (3, 600, 400), (1, 5000, 5000), (65535, 65535 * 7, 9), (64, 1 << 20, 1 << 15), (2, (1 << 31) - 2, 1 << 30)):
        for rules in (B.gta_score_rules(0.0), B.gta_score_rules(5.0, FAKE, FAKE, FAKE)):
            rc = B.load().gta_prefill_masked_attention(R(cfg), FAKE, q, FAKE, k, FAKE, c, FAKE, batch, total, longest, R(rules), FAKE, FAKE, (1 << 63) - 1, None)
            out.append([rc, events()])
""")
    assert _check(out)


def test_prefix_decode():
    out = S.run(SETUP + """
for name, dt, sh, cfg in cfgs():
    for batch in (1, 7, 64, 65, 300, 65535):
        for rows, own, page in ((1, 1, 0), (500, 1 << 14, 16), (1 << 30, 1 << 30, 0), (40000, 96, 32), (48, 48, 24)):
            up = lambda n: (n + max(page, 1) - 1) // max(page, 1) * max(page, 1)
            def cache(slots, n):
                n = up(n)
                return B.gta_cache(FAKE, FAKE, FAKE, FAKE, slots, n, FAKE if page else None, page, n // page if page else 0, 1 << 20)
            for rules in (None, B.gta_score_rules(5.0, FAKE, FAKE, FAKE)):
                rc = B.load().gta_prefix_decode_attention(R(cfg), FAKE, R(cache(1, rows)), 0, R(cache(batch, own)), None, batch, R(rules) if rules else None,
                                                          FAKE, FAKE, (1 << 63) - 1, None)
                out.append([rc, events()])
""")
    assert _check(out)
    for rc, text in out:   # the prefix, the own rows, the join; or the general kernel
        names = [e.kernel for e in S.parse(text) if isinstance(e, S.Launch)]
        assert rc or (len(names) == 1 and "prefix_any_kernel" in names[0]) or (
            len(names) == 3 and "rows_attn" in names[0] and "stream_kernel" in names[1] and "prefix_join_kernel" in names[2]), names


def test_workspaces_of_fuller_batches():
    """What gta_workspace_bytes says for a batch is enough for every smaller one."""
    out = S.run(SETUP + """
for name, dt, sh, cfg in cfgs():
    q, k, c = widths(sh)
    for rows, own in ((500, 1 << 12), (40000, 96)):
        for most in (40, 70, 300):
            n = B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFIX_DECODE, most, rows, own)
            caches = [B.gta_cache(FAKE, FAKE, FAKE, FAKE, 400, r, None, 0, 0, 0) for r in (rows, own)]
            for batch in (1, 2, 6, 7, 8, 12, 13, 16, 32, 33, 64, 65, 128, 129, 300):
                if batch <= most:
                    rc = B.load().gta_prefix_decode_attention(R(cfg), FAKE, R(caches[0]), 0, R(caches[1]), None, batch, None, FAKE, FAKE, n, None)
                    out.append([rc, [name, dt, most, batch]])
    for most in (3000, 20000):
        n = B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFILL_MASKED, 20, most, most)
        for total in (1, 100, 500, 1000, 1700, 2500, 4000, 6000, 8000, 10000, 15000, 20000):
            for batch in (1, 20):
                if total <= most:
                    rc = B.load().gta_prefill_masked_attention(R(cfg), FAKE, q, FAKE, k, FAKE, c, FAKE, batch, total, total, None, FAKE, FAKE, n, None)
                    out.append([rc, [name, dt, most, total]])
    events()
""")
    assert out and all(rc == 0 for rc, _ in out), [case for rc, case in out if rc]


def test_every_width_of_own_rows_has_its_kernel():
    out = S.run("""
for dh in (64, 128):
    for dl in range(64, 2049, 64):
        for nk in (1, 2, 3, 4, 5, 6, 7, 8, 11, 12, 16, 24, 64):
            for per in (1, 2, 5, 20):
                for nc in {1, 2, nk} if nk * per % 2 == 0 else {1, nk}:
                    if dl >= dh:
                        for dt in ("bf16", "f32"):
                            nq = nk * per
                            cfg = B.make_config(d_model=256, n_heads=nq, n_qgroups=nq, n_kgroups=nk, n_cgroups=nc, head_dim=dh, latent_dim=dl, dtype=dt)
                            cache = B.gta_cache(FAKE, FAKE, FAKE, FAKE, 5, 640)
                            rc = B.load().gta_prefix_decode_attention(R(cfg), FAKE, R(cache), 0, R(cache), None, 5, None, FAKE, FAKE, (1 << 63) - 1, None)
                            t = events()
                            out.append([rc, B.gta_uses_tuned_kernels(cfg, B.GTA_MODE_PREFIX_DECODE), nq, [t.count(n) for n in ("stream_kernel", "rows_attn", "prefix_join", "prefix_any")],
                                        sum(l.startswith("attr") and "stream_kernel" in l for l in t.splitlines())])
""")
    for rc, tuned, nq, (streams, rows, joins, general), attrs in out:
        assert rc == 0
        if tuned and nq <= 512:
            assert streams - attrs == 1 and rows >= 1 and joins == 1 and not general
        else:
            assert not streams and not joins and general == 1
    assert len(out) > 1000


def test_rotation():
    out = S.run(SETUP + """
for name, dt, sh, cfg in cfgs():
    q, k, c = widths(sh)
    for part in (0, 2, sh["head_dim"] // 2 // 2 * 2):
        rot = B.make_rotation(cfg, rotary_dim=part, layout="interleaved" if part else "half")
        for total in (1, 4000, 1 << 24, (1 << 31) // (sh["n_qgroups"] + sh["n_kgroups"]), (1 << 31) // (sh["n_qgroups"] + sh["n_kgroups"]) + 1):
            rc = B.load().gta_qk_rope(R(cfg), R(rot), FAKE, q, FAKE, k, None, total, 0, FAKE, q, FAKE, k, None)
            out.append([rc, events()])
""")
    for rc, text in out:
        ev = S.parse(text)
        assert (rc == -5 and not ev) or (rc == 0 and len(ev) == 1 and _fits(ev[0]))


def test_every_attention_kernel_is_run_by_some_layer_of_the_tests():
    """The kernels that the library has are the ones that the tests' layers, batches and rules take."""
    registered, taken = S.run(SETUP + """
taken = ""
for name, dt, sh, cfg in cfgs():
    q, k, c = widths(sh)
    for rules in (B.gta_score_rules(0.0), B.gta_score_rules(5.0), B.gta_score_rules(0.0, FAKE), B.gta_score_rules(5.0, FAKE)):
        assert B.load().gta_prefill_masked_attention(R(cfg), FAKE, q, FAKE, k, FAKE, c, FAKE, 2, 500, 2500, R(rules), FAKE, FAKE, (1 << 63) - 1, None) == 0
        taken += events()
        for batch in (1, 7, 9, 20, 33, 64, 65, 130):
            for rows in (512, 9216):
                prefix, own = B.gta_cache(FAKE, FAKE, FAKE, FAKE, 1, rows), B.gta_cache(FAKE, FAKE, FAKE, FAKE, batch, 256)
                assert B.load().gta_prefix_decode_attention(R(cfg), FAKE, R(prefix), 0, R(own), None, batch, R(rules), FAKE, FAKE, (1 << 63) - 1, None) == 0
                taken += events()
spy.spy_names.restype = ctypes.c_char_p
out += [spy.spy_names().decode().split(), taken]
""")
    mine = ("rows_attn_kernel", "rows_attn_f32_kernel", "stream_kernel", "prefix_join_kernel", "join_pieces_kernel", "plan_kernel", "masked_any_kernel",
            "prefix_any_kernel")
    other = ("proj_stream_kernel", "decoder_stream_kernel", "plain_stream_kernel")
    registered = {n for n in registered if any(m in n for m in mine) and not any(o in n for o in other)}
    taken = {e.kernel for e in S.parse(taken)}
    assert len(registered) > 60 and not registered - taken, sorted(registered - taken)
