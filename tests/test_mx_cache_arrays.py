"""Arrays that make_mx_cache and make_paged_mx_cache refuse: the kernels would read past their end, or something else than is
there.  No GPU: shapes and types are looked at on the host."""
import pytest
import torch

from paper_2506_17286_amd import binding as B


def arrays(paged=False, **kw):
    """Four slots of 64 rows, or 10 pages of 16 of them: one key of 64 and a latent of 128."""
    lead = (10, 16) if paged else (4, 64)
    a = dict(k=torch.zeros(*lead, 64, dtype=torch.uint8), c=torch.zeros(*lead, 128, dtype=torch.uint8),
             k_scale=torch.zeros(*lead, 2, dtype=torch.uint8), c_scale=torch.zeros(*lead, 4, dtype=torch.uint8),
             seq_lens=torch.zeros(4, dtype=torch.int32), status=torch.zeros(4, dtype=torch.int32))
    if paged:
        a["block_table"] = torch.zeros(4, 4, dtype=torch.int32)
    a.update(kw)
    return list(a.values())


BAD = {
    "scales of another width": dict(k_scale=(64,)), "a scale per 16 elements": dict(c_scale=(8,)), "codes of another width": dict(c=(96,)),
    "one scale a row": dict(c_scale=(1,)),
}


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("what", sorted(BAD))
def test_widths_that_do_not_belong_together(what, paged):
    make = B.make_paged_mx_cache if paged else B.make_mx_cache
    lead = (10, 16) if paged else (4, 64)
    (name, width), = BAD[what].items()
    with pytest.raises(ValueError):
        make(*arrays(paged, **{name: torch.zeros(*lead, *width, dtype=torch.uint8)}))


@pytest.mark.parametrize("paged", [False, True])
def test_other_refusals(paged):
    make = B.make_paged_mx_cache if paged else B.make_mx_cache
    lead = (10, 16) if paged else (4, 64)
    byte = dict(dtype=torch.uint8)
    bad = [dict(k=torch.zeros(*lead, 64, dtype=torch.bfloat16)), dict(k=torch.zeros(*lead, 64, dtype=torch.float8_e5m2)),
           dict(c_scale=torch.zeros(*lead, 4, dtype=torch.float32)), dict(c=torch.zeros(lead[0], lead[1] - 1, 128, **byte)),
           dict(c=torch.zeros(*lead, 256, **byte)[..., ::2]), dict(k=torch.zeros(lead[1], lead[0], 64, **byte).transpose(0, 1)),
           dict(k_scale=torch.zeros(lead[0] - 1, lead[1], 2, **byte)), dict(c_scale=torch.zeros(*lead, 4, device="meta", **byte)),
           dict(seq_lens=torch.zeros(4, dtype=torch.int64)), dict(status=torch.zeros(3, dtype=torch.int32)),
           dict(seq_lens=torch.zeros(3, dtype=torch.int32)), dict(status=torch.zeros(4, dtype=torch.int32, device="meta"))]
    if paged:
        bad += [dict(block_table=torch.zeros(4, 4, dtype=torch.int64)), dict(block_table=torch.zeros(4, 8, dtype=torch.int32)[:, ::2]),
                dict(block_table=torch.zeros(4, 4, dtype=torch.int32, device="meta")), dict(block_table=torch.zeros(5, 4, dtype=torch.int32))]
    for kw in bad:
        with pytest.raises(ValueError):
            make(*arrays(paged, **kw))


def test_what_is_taken():
    plain, paged = B.make_mx_cache(*arrays()), B.make_paged_mx_cache(*arrays(True))
    assert (plain.max_batch, plain.max_seq, plain.block_table) == (4, 64, None)
    assert (paged.max_batch, paged.max_seq, paged.page_size, paged.pages_per_slot, paged.num_pages) == (4, 64, 16, 4, 10)
    fp8 = [t.view(torch.float8_e4m3fn) if i < 2 else t for i, t in enumerate(arrays())]
    heads = arrays(k=torch.zeros(4, 64, 2, 32, dtype=torch.uint8), k_scale=torch.zeros(4, 64, 2, 1, dtype=torch.uint8))   # rows as heads
    longer = arrays(seq_lens=torch.zeros(9, dtype=torch.int32))
    for a in (fp8, heads, longer):
        cache = B.make_mx_cache(*a)
        assert cache.max_batch == 4 and cache.k == a[0].data_ptr() and cache.widths == (64, 128)


def test_calls_refuse_a_cache_of_another_device_or_layer(monkeypatch):
    """Before anything else is looked at: the current device is made up here, the library is not called."""
    monkeypatch.setattr(B, "_device", lambda: 0)
    monkeypatch.setattr(B, "load", lambda: pytest.fail("called"))
    monkeypatch.setattr(B, "_stream", lambda s: None)
    layer = dict(d_model=256, n_heads=4, n_qgroups=4, n_kgroups=1, n_cgroups=1, head_dim=64, dtype="bf16")
    cfg, other = B.make_config(latent_dim=128, **layer), B.make_config(latent_dim=256, **layer)
    on_host, there = B.make_mx_cache(*arrays()), B.make_mx_cache(*arrays())
    there.device = 0
    monkeypatch.setattr(B, "load", lambda: type("Lib", (), {n: staticmethod(lambda *a: pytest.fail("called")) for n in B.EXPORTS}))
    for c, cache in ((cfg, on_host), (other, there)):
        for call in (lambda: B.gta_mx_cache_append(c, cache, None, None, 64, None, 128, None, 1, 1),
                     lambda: B.gta_mx_cache_read(c, cache, None, None, None, 1, 1, None, None),
                     lambda: B.gta_mx_decode_attention(c, None, cache, None, 1, 0, None, None)):
            with pytest.raises(ValueError):
                call()
