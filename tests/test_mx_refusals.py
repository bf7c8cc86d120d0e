"""Arguments that the 8-bit cache and the query / key norm refuse on the host, before anything is enqueued.  No GPU."""
import ctypes

import pytest

from paper_2506_17286_amd import binding as B

FAKE = 4096   # never dereferenced: every call below is refused first
R = ctypes.byref


def _cfg(**kw):
    base = dict(d_model=256, n_heads=4, n_qgroups=4, n_kgroups=4, n_cgroups=1, head_dim=64, latent_dim=128, dtype="bf16")
    base.update(kw)
    return B.make_config(**base)


def _cache(**kw):
    f = dict(k=FAKE, c=FAKE, k_scale=FAKE, c_scale=FAKE, seq_lens=FAKE, status=FAKE, max_batch=2, max_seq=64, block_table=None,
             page_size=0, pages_per_slot=0, num_pages=0)
    f.update(kw)
    return B.gta_mx_cache(*f.values())


BAD_CACHES = [
    (dict(k=None), B.GTA_ERR_NULL), (dict(c=None), B.GTA_ERR_NULL), (dict(k_scale=None), B.GTA_ERR_NULL),
    (dict(c_scale=None), B.GTA_ERR_NULL), (dict(seq_lens=None), B.GTA_ERR_NULL), (dict(status=None), B.GTA_ERR_NULL),
    (dict(k=FAKE + 8), B.GTA_ERR_ALIGN), (dict(c_scale=FAKE + 1), B.GTA_ERR_ALIGN), (dict(k_scale=FAKE + 4), B.GTA_ERR_ALIGN),
    (dict(seq_lens=FAKE + 2), B.GTA_ERR_ALIGN), (dict(max_seq=0), B.GTA_ERR_SHAPE), (dict(max_batch=-1), B.GTA_ERR_SHAPE),
    (dict(block_table=FAKE, page_size=16, pages_per_slot=3, num_pages=8), B.GTA_ERR_SHAPE),
    (dict(block_table=FAKE, page_size=16, pages_per_slot=4, num_pages=0), B.GTA_ERR_SHAPE),
    (dict(block_table=FAKE + 2, page_size=16, pages_per_slot=4, num_pages=8), B.GTA_ERR_ALIGN),
]


def _append(cfg, cache, k=FAKE, ks=256, c=FAKE, cs=128, cu=FAKE, batch=1, most=1):
    return B.load().gta_mx_cache_append(R(cfg), R(cache) if cache else None, None, k, ks, c, cs, cu, batch, most, None)


def _read(cfg, cache, cu=FAKE, batch=1, most=1, k=FAKE, c=FAKE, first=None):
    return B.load().gta_mx_cache_read(R(cfg), R(cache) if cache else None, None, first, cu, batch, most, k, c, None)


def _attend(cfg, cache, q=FAKE, batch=1, splits=0, out=FAKE, ws=FAKE, size=1 << 30):
    return B.load().gta_mx_decode_attention(R(cfg), q, R(cache) if cache else None, None, batch, splits, out, ws, size, None)


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_bad_caches(kw, code):
    cfg, cache = _cfg(), _cache(**kw)
    assert _append(cfg, cache) == code
    assert _read(cfg, cache) == code
    assert _attend(cfg, cache) == code


@pytest.mark.parametrize("call", [_append, _read, _attend])
def test_widths_that_are_no_whole_blocks(call):
    for kw in (dict(head_dim=48), dict(latent_dim=144), dict(head_dim=16)):
        assert call(_cfg(**kw), _cache()) == B.GTA_ERR_UNSUPPORTED
    assert call(_cfg(dtype=5), _cache()) == B.GTA_ERR_DTYPE
    assert call(_cfg(), None) == B.GTA_ERR_NULL
    assert call(_cfg(), _cache(), batch=0) == B.GTA_ERR_SHAPE
    assert call(_cfg(), _cache(), batch=3) == B.GTA_ERR_SHAPE        # more sequences than slots
    assert call(_cfg(), _cache(max_batch=1 << 20), batch=65536) == B.GTA_ERR_SHAPE


def test_append_arguments():
    cfg, cache = _cfg(), _cache()
    assert _append(cfg, cache, k=None) == B.GTA_ERR_NULL
    assert _append(cfg, cache, c=None) == B.GTA_ERR_NULL
    assert _append(cfg, cache, cu=None) == B.GTA_ERR_NULL
    assert _append(cfg, cache, ks=255) == B.GTA_ERR_SHAPE            # rows would overlap
    assert _append(cfg, cache, cs=-128) == B.GTA_ERR_SHAPE
    assert _append(cfg, cache, cs=1 << 40) == B.GTA_ERR_SHAPE
    assert _append(cfg, cache, most=-1) == B.GTA_ERR_SHAPE
    assert _append(cfg, cache, k=FAKE + 1) == B.GTA_ERR_ALIGN
    assert _append(_cfg(dtype="f32"), cache, c=FAKE + 2) == B.GTA_ERR_ALIGN
    assert _append(cfg, cache, cu=FAKE + 2) == B.GTA_ERR_ALIGN


def test_read_arguments():
    cfg, cache = _cfg(), _cache()
    assert _read(cfg, cache, k=None) == B.GTA_ERR_NULL
    assert _read(cfg, cache, cu=None) == B.GTA_ERR_NULL
    assert _read(cfg, cache, c=FAKE + 8) == B.GTA_ERR_ALIGN
    assert _read(cfg, cache, first=FAKE + 2) == B.GTA_ERR_ALIGN
    assert _read(cfg, cache, most=-1) == B.GTA_ERR_SHAPE
    assert _read(cfg, cache, most=0) == B.GTA_OK                     # nothing to read


def test_attention_arguments():
    cfg, cache = _cfg(), _cache()
    assert _attend(cfg, cache, q=None) == B.GTA_ERR_NULL
    assert _attend(cfg, cache, out=None) == B.GTA_ERR_NULL
    assert _attend(cfg, cache, splits=-1) == B.GTA_ERR_SHAPE
    assert _attend(cfg, cache, q=FAKE + 2) == B.GTA_ERR_ALIGN
    assert _attend(cfg, cache, ws=None) == B.GTA_ERR_WORKSPACE
    assert _attend(cfg, cache, ws=FAKE + 8) == B.GTA_ERR_WORKSPACE
    assert _attend(cfg, cache, size=16) == B.GTA_ERR_WORKSPACE
    need = B.gta_workspace_bytes(cfg, B.GTA_MODE_MX_DECODE, 1, 0, 64, 8)
    assert _attend(cfg, cache, splits=8, size=need // 2) == B.GTA_ERR_WORKSPACE
    assert _attend(_cfg(head_dim=2048, latent_dim=2048), cache) == B.GTA_ERR_UNSUPPORTED
    assert _attend(_cfg(latent_dim=8192), cache) == B.GTA_ERR_UNSUPPORTED


def test_workspace_sizes():
    cfg = _cfg()
    size = lambda b, n, s=0: B.gta_workspace_bytes(cfg, B.GTA_MODE_MX_DECODE, b, 0, n, s)   # noqa: E731
    assert 0 < size(4, 4096, 1) < size(4, 4096, 8)
    assert size(4, 4096) >= size(4, 4096, 1)
    assert size(65535, (1 << 31) - 1, 1024) > 0
    assert size(1, 64, -1) == 0 and size(0, 64) == 0
    assert B.gta_workspace_bytes(_cfg(head_dim=48), B.GTA_MODE_MX_DECODE, 1, 0, 64) == 0


def test_norm_arguments():
    def call(cfg=None, q=FAKE, qs=256, k=FAKE, ks=256, qg=None, kg=None, eps=1e-6, pos=None, n=1, qo=FAKE, ko=FAKE):
        return B.load().gta_qk_norm_rope(R(cfg or _cfg()), q, qs, k, ks, qg, kg, eps, pos, n, qo, ko, None)

    for name in ("q", "k", "qo", "ko"):
        assert call(**{name: None}) == B.GTA_ERR_NULL
    assert call(n=-1) == B.GTA_ERR_SHAPE and call(n=1 << 31) == B.GTA_ERR_SHAPE
    for eps in (-1e-6, float("nan"), float("inf")):
        assert call(eps=eps) == B.GTA_ERR_SHAPE
    assert call(qs=255) == B.GTA_ERR_SHAPE and call(ks=-256) == B.GTA_ERR_SHAPE and call(ks=1 << 40) == B.GTA_ERR_SHAPE
    assert call(q=FAKE + 1) == B.GTA_ERR_ALIGN and call(kg=FAKE + 1) == B.GTA_ERR_ALIGN
    assert call(cfg=_cfg(dtype="f32"), k=FAKE + 2) == B.GTA_ERR_ALIGN
    assert call(qo=FAKE + 8) == B.GTA_ERR_ALIGN and call(pos=FAKE + 2) == B.GTA_ERR_ALIGN
    assert call(cfg=_cfg(head_dim=63, rope=True)) == B.GTA_ERR_SHAPE
    assert call(n=0) == B.GTA_OK                                     # nothing to do


def test_struct_layout():
    assert ctypes.sizeof(B.gta_mx_cache) == 6 * 8 + 2 * 4 + 8 + 3 * 4 + 4
    assert B.gta_mx_cache.block_table.offset == 56 and B.gta_mx_cache.num_pages.offset == 72


@pytest.mark.parametrize("dims,answer", [
    ((4, 4, 1, 128, 512), 1), ((8, 8, 1, 128, 1024), 1), ((5, 1, 1, 64, 128), 1), ((10, 1, 2, 64, 128), 1), ((4, 4, 4, 128, 512), 1),
    ((2, 1, 1, 256, 256), 1), ((2, 2, 1, 32, 64), 1), ((20, 20, 20, 64, 64), 1), ((6, 3, 2, 96, 160), 1), ((32, 1, 1, 64, 128), 1),
    ((2, 1, 1, 512, 1024), 1), ((2, 1, 1, 544, 544), 0), ((4096, 1, 1, 32, 32), 1),
    ((2, 1, 1, 48, 128), B.GTA_ERR_UNSUPPORTED), ((1, 1, 1, 2048, 2048), B.GTA_ERR_UNSUPPORTED)])
def test_which_kernel(dims, answer):
    nq, nk, nc, dh, dl = dims
    for dtype in ("bf16", "f32"):
        cfg = _cfg(n_heads=nq, n_qgroups=nq, n_kgroups=nk, n_cgroups=nc, head_dim=dh, latent_dim=dl, dtype=dtype)
        assert B.gta_uses_tuned_kernels(cfg, B.GTA_MODE_MX_DECODE) == answer


def test_slots_of_more_rows_than_row_numbers_take():
    table = dict(block_table=FAKE, page_size=1 << 15, num_pages=1 << 20)
    for seq, batch in (((1 << 31) - (1 << 15), 1), (1 << 30, 64), (1 << 27, 512)):
        cache = _cache(max_seq=seq, pages_per_slot=seq >> 15, max_batch=1024, **table)
        assert _attend(_cfg(), cache, batch=batch, size=1 << 40) == B.GTA_ERR_UNSUPPORTED
