"""Arguments that the rotation and the attention with rules refuse on the host, before anything is enqueued.  No GPU."""
import ctypes
import math

import pytest

import rules_util as U
from paper_2506_17286_amd import binding as B

FAKE = 4096   # never dereferenced: every call below is refused first
R = ctypes.byref


def _cfg(**kw):
    base = dict(d_model=256, n_heads=4, n_qgroups=4, n_kgroups=4, n_cgroups=1, head_dim=64, latent_dim=128, dtype="bf16")
    base.update(kw)
    return B.make_config(**base)


def _spec(**kw):
    base = dict(layout=0, rotary_dim=0, scaling=0, base=10000.0, factor=1.0, trained_len=0.0, slow_turns=0.0, fast_turns=0.0, magnitude=0.0, frequency=None)
    base.update(kw)
    return B.gta_rope_spec(*base.values())


BANDS = dict(scaling=3, factor=8.0, trained_len=4096.0, slow_turns=1.0, fast_turns=4.0)


@pytest.mark.parametrize("kw,code", [
    (dict(), 0), (dict(layout=1), 0), (BANDS, 0), (dict(scaling=1, factor=0.5), 0), (dict(rotary_dim=2), 0),
    (dict(layout=2), B.GTA_ERR_DTYPE), (dict(scaling=5), B.GTA_ERR_DTYPE), (dict(scaling=-1), B.GTA_ERR_DTYPE),
    (dict(rotary_dim=3), B.GTA_ERR_SHAPE), (dict(rotary_dim=66), B.GTA_ERR_SHAPE), (dict(rotary_dim=-2), B.GTA_ERR_SHAPE),
    (dict(base=0.0), B.GTA_ERR_SHAPE), (dict(base=math.nan), B.GTA_ERR_SHAPE), (dict(base=math.inf), B.GTA_ERR_SHAPE),
    (dict(magnitude=-1.0), B.GTA_ERR_SHAPE), (dict(magnitude=math.nan), B.GTA_ERR_SHAPE),
    (dict(scaling=1, factor=0.0), B.GTA_ERR_SHAPE), (dict(scaling=2, factor=math.inf), B.GTA_ERR_SHAPE), (dict(scaling=2, factor=2.0, rotary_dim=2), B.GTA_ERR_SHAPE),
    (dict(BANDS, trained_len=0.0), B.GTA_ERR_SHAPE), (dict(BANDS, slow_turns=4.0), B.GTA_ERR_SHAPE), (dict(BANDS, fast_turns=math.nan), B.GTA_ERR_SHAPE),
    (dict(scaling=4), B.GTA_ERR_NULL),
])
def test_rotation_specs(kw, code):
    out = B.gta_rotation()
    cfg = _cfg()
    assert B.load().gta_make_rotation(R(cfg), R(_spec(**kw)), R(out)) == code
    if code == 0:
        assert out.rotary_dim == (kw.get("rotary_dim") or 64) and out.magnitude == 1.0 and out.layout == kw.get("layout", 0)
    else:
        assert out.rotary_dim == 0     # nothing written
    assert B.load().gta_make_rotation(None, R(_spec()), R(out)) == B.GTA_ERR_NULL
    assert B.load().gta_make_rotation(R(cfg), None, R(out)) == B.GTA_ERR_NULL
    assert B.load().gta_make_rotation(R(cfg), R(_spec()), None) == B.GTA_ERR_NULL


def test_rotation_of_more_pairs_than_there_is_room_for():
    cfg, out = _cfg(head_dim=1024, latent_dim=1024), B.gta_rotation()
    assert B.load().gta_make_rotation(R(cfg), R(_spec()), R(out)) == B.GTA_ERR_UNSUPPORTED
    assert B.load().gta_make_rotation(R(cfg), R(_spec(rotary_dim=512)), R(out)) == 0


def test_given_frequencies():
    cfg = _cfg()
    with pytest.raises(ValueError):
        B.make_rotation(cfg, scaling="given", frequencies=[1.0] * 31)
    for bad in (math.nan, math.inf, -math.inf, 1e30):
        with pytest.raises(B.GtaError):
            B.make_rotation(cfg, scaling="given", frequencies=[1.0] * 31 + [bad])
    rot = B.make_rotation(cfg, scaling="given", frequencies=[math.pi, -math.pi / 2] + [0.0] * 30)
    assert abs(rot.turn[0] - 2 ** 63) < 2 ** 13 and abs(rot.turn[1] - 3 * 2 ** 62) < 2 ** 13 and rot.turn[2] == 0


def test_turns_of_a_plain_rotation():
    """base^(-2j/r) / (2 pi) in units of 2^-64, against 80 decimal digits."""
    from decimal import Decimal, getcontext
    getcontext().prec = 80
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")
    for base in (10000.0, 500000.0):
        rot = B.make_rotation(_cfg(head_dim=128, latent_dim=128), base=base)
        for j in (0, 1, 17, 63):
            want = (Decimal(base).ln() * Decimal(-2 * j) / 128).exp() / (2 * pi) * 2 ** 64
            assert abs(Decimal(rot.turn[j]) - want) <= 64      # 2^-58 of a turn: 2^-27 at the last position there is


def _rope(cfg, rot, q=FAKE, qs=256, k=FAKE, ks=256, pos=None, n=4, back=0, qo=FAKE, qos=256, ko=FAKE, kos=256):
    return B.load().gta_qk_rope(R(cfg), R(rot) if rot else None, q, qs, k, ks, pos, n, back, qo, qos, ko, kos, None)


def test_rope_arguments():
    cfg = _cfg()
    rot = B.make_rotation(cfg)
    assert _rope(cfg, None) == B.GTA_ERR_NULL
    assert _rope(cfg, rot, q=None) == B.GTA_ERR_NULL                  # an output without its input
    assert _rope(cfg, rot, ko=None) == B.GTA_ERR_NULL
    assert _rope(cfg, rot, q=None, qo=None, k=None, ko=None) == B.GTA_ERR_NULL
    assert _rope(cfg, rot, qs=255) == B.GTA_ERR_SHAPE
    assert _rope(cfg, rot, kos=-256) == B.GTA_ERR_SHAPE
    assert _rope(cfg, rot, ks=1 << 40) == B.GTA_ERR_SHAPE
    assert _rope(cfg, rot, qs=512) == B.GTA_ERR_SHAPE                 # in place with another stride
    assert _rope(cfg, rot, n=-1) == B.GTA_ERR_SHAPE
    assert _rope(cfg, rot, n=1 << 31) == B.GTA_ERR_SHAPE
    assert _rope(cfg, rot, n=1 << 30) == B.GTA_ERR_UNSUPPORTED
    assert _rope(cfg, rot, q=FAKE + 1, qo=2 * FAKE) == B.GTA_ERR_ALIGN
    assert _rope(cfg, rot, pos=FAKE + 2) == B.GTA_ERR_ALIGN
    assert _rope(cfg, rot, back=2) == B.GTA_ERR_DTYPE
    wide = B.make_rotation(_cfg(head_dim=128, latent_dim=128))
    assert _rope(cfg, wide) == B.GTA_ERR_SHAPE                        # of wider heads
    for field, value, code in (("layout", 9, B.GTA_ERR_DTYPE), ("rotary_dim", 0, B.GTA_ERR_SHAPE), ("magnitude", math.nan, B.GTA_ERR_SHAPE)):
        other = B.make_rotation(cfg)
        setattr(other, field, value)
        assert _rope(cfg, other) == code


def _masked(cfg, q=FAKE, qs=256, k=FAKE, ks=256, c=FAKE, cs=128, cu=None, batch=1, total=4, longest=4, rules=None, out=FAKE, ws=FAKE, size=1 << 40):
    return B.load().gta_prefill_masked_attention(R(cfg), q, qs, k, ks, c, cs, cu, batch, total, longest, R(rules) if rules else None, out, ws, size, None)


def _cache(**kw):
    f = dict(k=FAKE, c=FAKE, seq_lens=FAKE, status=FAKE, max_batch=2, max_seq=64, block_table=None, page_size=0, pages_per_slot=0, num_pages=0)
    f.update(kw)
    return B.gta_cache(*f.values())


def _prefix(cfg, q=FAKE, prefix=None, slot=0, cache=None, batch=1, rules=None, out=FAKE, ws=FAKE, size=1 << 40, slots=None):
    prefix, cache = prefix or _cache(), cache or _cache()
    return B.load().gta_prefix_decode_attention(R(cfg), q, R(prefix), slot, R(cache), slots, batch, R(rules) if rules else None, out, ws, size, None)


@pytest.mark.parametrize("call", [_masked, _prefix])
def test_rules_of_either_attention(call):
    cfg = _cfg()
    for cap in (-1.0, math.nan, math.inf, 1e-31, 1e-40, 2e30):
        assert call(cfg, rules=B.gta_score_rules(cap)) == B.GTA_ERR_SHAPE
    for field in ("slopes", "first", "last"):
        rules = B.gta_score_rules(0.0)
        setattr(rules, field, FAKE + 2)
        assert call(cfg, rules=rules) == B.GTA_ERR_ALIGN
    assert call(_cfg(dtype=7)) == B.GTA_ERR_DTYPE
    assert call(_cfg(n_kgroups=3)) == B.GTA_ERR_SHAPE
    assert call(cfg, q=None) == B.GTA_ERR_NULL
    assert call(cfg, out=None) == B.GTA_ERR_NULL
    assert call(cfg, out=FAKE + 8) == B.GTA_ERR_ALIGN
    assert call(cfg, ws=None) == B.GTA_ERR_WORKSPACE
    assert call(cfg, ws=FAKE + 4) == B.GTA_ERR_WORKSPACE
    assert call(cfg, batch=0) == B.GTA_ERR_SHAPE
    assert call(cfg, batch=65536) == B.GTA_ERR_SHAPE
    assert call(_cfg(head_dim=1026, latent_dim=1026), **({} if call is _prefix else dict(qs=8192, ks=8192, cs=8192))) == B.GTA_ERR_UNSUPPORTED
    assert call(_cfg(latent_dim=4100), **({} if call is _prefix else dict(cs=8192))) == B.GTA_ERR_UNSUPPORTED


def test_masked_arguments():
    cfg = _cfg()
    assert _masked(cfg, k=None) == B.GTA_ERR_NULL
    assert _masked(cfg, c=None) == B.GTA_ERR_NULL
    assert _masked(cfg, qs=255) == B.GTA_ERR_SHAPE
    assert _masked(cfg, ks=-256) == B.GTA_ERR_SHAPE
    assert _masked(cfg, cs=127) == B.GTA_ERR_SHAPE
    assert _masked(cfg, cs=1 << 40) == B.GTA_ERR_SHAPE
    assert _masked(cfg, total=-1) == B.GTA_ERR_SHAPE
    assert _masked(cfg, total=1 << 31) == B.GTA_ERR_SHAPE
    assert _masked(cfg, batch=3) == B.GTA_ERR_SHAPE                   # 4 tokens in 3 equal sequences
    assert _masked(cfg, longest=3) == B.GTA_ERR_SHAPE
    assert _masked(cfg, longest=-1) == B.GTA_ERR_SHAPE
    assert _masked(cfg, q=FAKE + 1) == B.GTA_ERR_ALIGN
    assert _masked(_cfg(dtype="f32"), c=FAKE + 2) == B.GTA_ERR_ALIGN
    assert _masked(cfg, cu=FAKE + 2) == B.GTA_ERR_ALIGN
    assert _masked(cfg, total=0, longest=0) == 0                      # nothing to do


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), B.GTA_ERR_NULL), (dict(c=None), B.GTA_ERR_NULL), (dict(seq_lens=None), B.GTA_ERR_NULL), (dict(status=None), B.GTA_ERR_NULL),
    (dict(k=FAKE + 8), B.GTA_ERR_ALIGN), (dict(seq_lens=FAKE + 2), B.GTA_ERR_ALIGN), (dict(max_seq=0), B.GTA_ERR_SHAPE),
    (dict(max_batch=-1), B.GTA_ERR_SHAPE), (dict(max_seq=(1 << 30) + 1), B.GTA_ERR_UNSUPPORTED),
    (dict(block_table=FAKE, page_size=16, pages_per_slot=3, num_pages=8), B.GTA_ERR_SHAPE),
    (dict(block_table=FAKE + 2, page_size=16, pages_per_slot=4, num_pages=8), B.GTA_ERR_ALIGN),
])
def test_prefix_caches(kw, code):
    assert _prefix(_cfg(), prefix=_cache(**kw)) == code
    assert _prefix(_cfg(), cache=_cache(**kw)) == code


def test_prefix_arguments():
    cfg = _cfg()
    assert _prefix(cfg, batch=3) == B.GTA_ERR_SHAPE                   # more sequences than slots
    assert _prefix(cfg, slot=-1) == B.GTA_ERR_SHAPE
    assert _prefix(cfg, slot=2) == B.GTA_ERR_SHAPE
    assert _prefix(cfg, slots=FAKE + 2) == B.GTA_ERR_ALIGN
    assert _prefix(cfg, q=FAKE + 8) == B.GTA_ERR_ALIGN
    assert B.load().gta_prefix_decode_attention(R(cfg), FAKE, None, 0, R(_cache()), None, 1, None, FAKE, FAKE, 1 << 40, None) == B.GTA_ERR_NULL
    assert B.load().gta_prefix_decode_attention(R(cfg), FAKE, R(_cache()), 0, None, None, 1, None, FAKE, FAKE, 1 << 40, None) == B.GTA_ERR_NULL


@pytest.mark.parametrize("mode", [B.GTA_MODE_PREFILL_MASKED, B.GTA_MODE_PREFIX_DECODE])
def test_workspaces(mode):
    cfg = _cfg()
    for batch, total, longest in ((1, 1, 1), (4, 4000, 1000), (65535, 1 << 20, 1 << 10), (1, 1 << 30, 1 << 30)):
        n = B.gta_workspace_bytes(cfg, mode, batch, total, longest)
        assert n > 0
        call = _masked if mode == B.GTA_MODE_PREFILL_MASKED else _prefix
        kw = dict(batch=batch, total=total, longest=longest, cu=FAKE) if call is _masked else dict(
            batch=batch, prefix=_cache(max_seq=total), cache=_cache(max_seq=longest, max_batch=65535))
        if n > 256:
            assert call(cfg, size=0, **kw) == B.GTA_ERR_WORKSPACE
    assert B.gta_workspace_bytes(cfg, mode, 0, 1, 1) == 0
    assert B.gta_workspace_bytes(cfg, mode, 1, -1, 1) == 0
    assert B.gta_workspace_bytes(cfg, mode, 1, 1, -1) == 0
    assert B.gta_workspace_bytes(_cfg(latent_dim=4100), mode, 1, 1, 1) == 0
    assert B.gta_uses_tuned_kernels(_cfg(latent_dim=4100), mode) == B.GTA_ERR_UNSUPPORTED


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", sorted(U.SHAPES))
def test_a_workspace_does_for_fewer_sequences_and_tokens(name, dtype):
    cfg = U.config(name, dtype)
    for rows, own in ((0, 0), (1, 1), (500, 4096), (8192, 100), (40000, 1 << 20)):
        sizes = [B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFIX_DECODE, b, rows, own) for b in [*range(1, 300), 400, 511, 512, 1000, 3000, 65535]]
        assert sizes == sorted(sizes), (rows, own)
    totals = [1, 2, 31, 100, 1000, *range(1500, 9000, 250), 10000, 20000, 40000, 1 << 20]
    for batch in (1, 2, 30, 300, 3000):
        sizes = [B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFILL_MASKED, batch, t, t) for t in totals]
        assert sizes == sorted(sizes), batch
    for t in totals:
        sizes = [B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFILL_MASKED, b, t, t) for b in (1, 2, 7, 30, 64, 100, 200, 300, 3000)]
        assert sizes == sorted(sizes), t


def test_binding_looks_at_tensors():
    import torch
    cfg = _cfg()
    with pytest.raises(ValueError):
        B.make_score_rules(slopes=torch.zeros(4, dtype=torch.float64))
    with pytest.raises(ValueError):
        B.make_score_rules(first=torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError):
        B.make_score_rules(last=torch.zeros(8, dtype=torch.int32)[::2])
    rules = B.make_score_rules(first=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        B._rules(-1, cfg, rules, 4)                     # fewer than there are tokens
    with pytest.raises(ValueError):
        B._rules(0, cfg, rules, 3)                      # on the host
    k, c = torch.zeros(2, 64, 256, dtype=torch.bfloat16), torch.zeros(2, 64, 128, dtype=torch.bfloat16)
    n = torch.zeros(2, dtype=torch.int32)
    cache = B.make_cache(k, c, n, n)
    assert B._rows_of(-1, cfg, cache) is not None
    for bad, kw in ((cache, dict(latent_dim=256)), (B.make_cache(k.float(), c.float(), n, n), {}), (B.make_cache(k, c[..., :64], n, n), {})):
        with pytest.raises(ValueError):
            B._rows_of(-1, _cfg(**kw), bad)
    with pytest.raises(ValueError):
        B._rows_of(0, cfg, cache)                       # on the host
