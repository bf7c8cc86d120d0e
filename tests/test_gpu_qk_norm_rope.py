"""gta_qk_norm_rope against the formula in float64: head widths on and off the vector kernel's grid, strided and unaligned
rows, far positions, gains or none, in place, one token to many."""
import numpy as np
import pytest
import torch

from paper_2506_17286_amd import binding as B

import mx_util as M

pytestmark = pytest.mark.gpu


def run(sh, dtype, tokens, pos, *, rope=True, base=10000.0, gains=True, fused=0, offset=0, eps=1e-6, seed=0, in_place=False, x=None):
    """fused: extra columns between the rows; offset: elements the first row is moved by."""
    rng = np.random.default_rng(seed)
    dt, dh = M.DT[dtype], sh["head_dim"]
    qw, kw = sh["n_qgroups"] * dh, sh["n_kgroups"] * dh
    cfg = B.make_config(dtype=dtype, rope=rope, rope_base=base, **sh)
    if x is None:
        x = rng.standard_normal((tokens, qw + kw)) * np.exp(rng.standard_normal((tokens, 1)))
    if in_place or not (fused or offset):
        q, k = (torch.from_numpy(v.copy()).to("cuda", dt) for v in (x[:, :qw], x[:, qw:]))
    else:
        buf = torch.zeros(offset + tokens * (qw + kw + fused), dtype=dt, device="cuda")[offset:].view(tokens, qw + kw + fused)
        buf[:, :qw + kw] = torch.from_numpy(x).to("cuda", dt)
        q, k = buf[:, :qw], buf[:, qw:qw + kw]
    gq, gk = ((torch.from_numpy(1 + 0.3 * rng.standard_normal(dh)).to("cuda", dt) if gains else None) for _ in range(2))
    p = None if pos is None else torch.tensor(pos, dtype=torch.int32, device="cuda")
    guard = 7.0
    qo, ko = (torch.full((tokens + 1, w), guard, dtype=dt, device="cuda") for w in (qw, kw))
    src = [t.double().cpu().numpy() for t in (q, k)]
    if in_place:
        qo[:tokens], ko[:tokens] = q, k
        q, k = qo, ko
    B.gta_qk_norm_rope(cfg, q, q.stride(0), k, k.stride(0), gq, gk, eps, p, tokens, qo, ko)
    torch.cuda.synchronize()
    assert (qo[tokens] == guard).all() and (ko[tokens] == guard).all()
    where = np.arange(tokens) if pos is None else np.asarray(pos)
    for got, v, g in ((qo, src[0], gq), (ko, src[1], gk)):
        ref, mag = M.norm_rope(v, None if g is None else g.double().cpu().numpy(), eps, where, dh, float(np.float32(base)), rope)
        got = got[:tokens].double().cpu().numpy()
        # fp32 roundings: the sum of squares (at most 22 in a row, halved by the root), mean, root, norm, gain, sine (1.0),
        # and the rotation's products and sum: 19 half steps of the rotated pair's length, counted as 32; then one of the result
        err = 32 * 2.0 ** -24 * mag
        bound = err + M.HALF_STEP[dtype] * (np.abs(ref) + err)
        worst = (np.abs(got - ref) / np.maximum(bound, 1e-300)).max()
        assert worst <= 1, f"{worst:.2f} of the bound"
    return qo, ko


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["paper", "1b", "wide", "tiny", "odd", "head256", "gta4", "mha"])
@pytest.mark.parametrize("tokens", [1, 3, 64, 257])
def test_layers(name, dtype, tokens):
    pos = np.random.default_rng(tokens).integers(0, 40000, tokens)
    run(M.SHAPES[name], dtype, tokens, pos, seed=tokens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,rope", [(2, True), (6, True), (20, True), (34, True), (48, True), (63, False), (1, False), (128, False), (320, True), (512, True), (1000, True)])
def test_head_widths(dh, rope, dtype):
    run(M.shape(3, 1, 1, dh, max(dh, 32)), dtype, 37, np.arange(37) * 11, rope=rope, seed=dh)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fused,offset", [(64, 0), (7, 0), (1, 0), (64, 1), (0, 2), (0, 8)])
def test_strides_and_alignment(fused, offset, dtype):
    run(M.SHAPES["1b"], dtype, 65, np.arange(65), fused=fused, offset=offset)
    run(M.SHAPES["paper"], dtype, 3, None, fused=fused, offset=offset)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["1b", "paper", "odd"])
def test_in_place(name, dtype):
    run(M.SHAPES[name], dtype, 130, np.arange(130) + 5, in_place=True)


@pytest.mark.parametrize("name", ["1b", "odd"])
def test_far_positions_and_bases(name):
    pos = [0, 1, 131071, 1 << 20, (1 << 31) - 1, -1, -5000]
    for base in (10000.0, 500000.0, 1.0, 0.5):
        run(M.SHAPES[name], "f32", len(pos), pos, base=base)
    run(M.SHAPES[name], "bf16", len(pos), pos, base=500000.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_gain_no_positions_and_large_eps(dtype):
    run(M.SHAPES["1b"], dtype, 50, None, gains=False, eps=0.0)
    run(M.SHAPES["1b"], dtype, 50, None, gains=False, eps=2.0)
    run(M.SHAPES["1b"], dtype, 50, None, rope=False)


@pytest.mark.parametrize("name", ["1b", "odd"])
def test_zero_rows_and_values_that_are_not_finite(name):
    sh = M.SHAPES[name]
    dh, w = sh["head_dim"], (sh["n_qgroups"] + sh["n_kgroups"]) * sh["head_dim"]
    run(sh, "bf16", 4, None, x=np.zeros((4, w)))
    x = np.random.default_rng(0).standard_normal((5, w))
    bad = x.copy()
    bad[2, dh + 3] = np.nan
    cfg = B.make_config(dtype="f32", rope=True, **sh)
    qw = sh["n_qgroups"] * dh
    outs = []
    for v in (x, bad):
        t = torch.from_numpy(v).float().cuda()
        qo, ko = torch.empty(5, qw, device="cuda"), torch.empty(5, w - qw, device="cuda")
        B.gta_qk_norm_rope(cfg, t, w, t[:, qw:], w, None, None, 1e-6, None, 5, qo, ko)
        outs.append(torch.cat([qo, ko], dim=1).cpu())
    hit = torch.zeros(5, w, dtype=torch.bool)
    hit[2, dh:2 * dh] = True                              # the head with the NaN, and nothing else
    assert torch.isnan(outs[1][hit]).all() and torch.equal(outs[0][~hit], outs[1][~hit])


def test_many_tokens_across_2_31_elements():
    """Rows whose element offset passes 32 bits."""
    sh, tokens, stride = M.SHAPES["paper"], 70, 1 << 25
    dh = sh["head_dim"]
    buf = torch.zeros(tokens * stride + 4096, dtype=torch.bfloat16, device="cuda")
    rows = buf[:tokens * stride].view(tokens, stride)
    rows[:, :6 * dh] = torch.randn(tokens, 6 * dh, generator=torch.Generator().manual_seed(0)).to("cuda", torch.bfloat16)
    cfg = B.make_config(dtype="bf16", rope=True, **sh)
    outs = []
    for src, st in ((rows, stride), (rows[:, :6 * dh].contiguous(), 6 * dh)):
        qo, ko = (torch.empty(tokens, n * dh, dtype=torch.bfloat16, device="cuda") for n in (5, 1))
        B.gta_qk_norm_rope(cfg, src, st, src[:, 5 * dh:], st, None, None, 1e-6, None, tokens, qo, ko)
        outs += [qo, ko]
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])


def test_more_rows_than_a_launch_has_workgroups():
    """4.5 million heads off the vector kernel's grid: workgroups go on to further ones."""
    run(M.shape(2, 1, 1, 6, 32), "f32", 1_500_000, None, rope=True, base=500000.0)
