"""gta_qk_rope against the rotation in extended precision: layouts, parts of the head, scalings, strides, directions."""
import numpy as np
import pytest
import torch

import rules_util as R
from paper_2506_17286_amd import binding as B

pytestmark = pytest.mark.gpu

BANDS = dict(scaling="bands", factor=8.0, trained_len=4096.0, slow_turns=1.0, fast_turns=4.0)


def _run(name, dtype, total, *, layout="half", part=None, spec=None, positions=None, transposed=False, magnitude=1.0, pad=0, offset=0,
         in_place=False, seed=1, out_pad=0, sides="qk"):
    """Rotates random rows (pad: elements between rows, offset: elements in front of the first) and checks every element."""
    cfg = R.config(name, dtype)
    sh, dh, dt = R.SHAPES[name], R.SHAPES[name]["head_dim"], R.DT[dtype]
    r = part or dh
    spec = dict(spec or {})
    rot = B.make_rotation(cfg, layout=layout, rotary_dim=r, magnitude=magnitude, **spec)
    spec["given"] = spec.pop("frequencies", None)
    gen = R.generator(seed)
    pos = None if positions is None else torch.tensor(positions, dtype=torch.int32, device="cuda")
    sides_out, tensors = {}, {}
    for side, heads in (("q", sh["n_qgroups"]), ("k", sh["n_kgroups"])):
        w = heads * dh
        flat = R.rows(gen, 1, offset + total * (w + pad), dtype)[0]
        x = flat[offset:].view(total, w + pad)
        out = x if in_place else torch.full((total, w + out_pad), float("nan"), dtype=dt, device="cuda")
        tensors[side] = (x, w, heads, x.clone(), out)
    args = []
    for side in "qk":
        x, w, heads, before, out = tensors[side]
        args.append((x, x.stride(0), out, out.stride(0)) if side in sides else (None, 0, None, 0))
    B.gta_qk_rope(cfg, rot, args[0][0], args[0][1], args[1][0], args[1][1], pos, total, transposed, args[0][2], args[0][3], args[1][2], args[1][3])
    torch.cuda.synchronize()
    freq = R.frequencies(r, **spec)
    p = np.arange(total) if positions is None else np.asarray(positions, dtype=np.int64)
    for side in sides:
        x, w, heads, before, out = tensors[side]
        ref, size = R.rotate(before[:, :w].double().cpu().numpy(), heads, dh, r, freq, p, layout == "interleaved", transposed, magnitude)
        got = out[:, :w].double().cpu().numpy()
        # sines: within 1e-7 (bf16 rows) or half a step of fp32; a sum of two products, the magnitude: four roundings of fp32
        loose = (1.0e-7 if dtype == "bf16" else 2.0 ** -24) + 4 * 2.0 ** -24
        tol = R.HALF_STEP[dtype] * np.abs(ref) + loose * size * (1 + R.HALF_STEP[dtype])
        assert np.all(np.abs(got - ref) <= tol), f"{side}: {np.max(np.abs(got - ref) / np.maximum(tol, 1e-300)):.2f} of the bound"
        if r < dh:
            same = out[:, :w].reshape(total, heads, dh)[..., r:]
            assert torch.equal(same, before[:, :w].reshape(total, heads, dh)[..., r:])
        if out_pad:
            assert bool(torch.isnan(out[:, w:]).all())
        if in_place and pad:
            assert torch.equal(out[:, w:], before[:, w:])
        sides_out[side] = out
    return sides_out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("name,part", [("1b", None), ("1b", 64), ("paper", None), ("paper", 16), ("odd", None), ("odd", 6), ("h96", 32),
                                       ("h32", 2), ("h32", None), ("1b", 96), ("1b", 24), ("h96", None)])
def test_layouts_and_parts(name, part, layout, dtype):
    for total in (1, 3, 70):
        _run(name, dtype, total, layout=layout, part=part, positions=[(i * 37) % 5000 for i in range(total)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("spec", [dict(), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0), BANDS,
                                  dict(BANDS, trained_len=128.0, slow_turns=0.25, fast_turns=32.0), dict(base=500000.0), dict(base=0.5),
                                  dict(scaling="given", frequencies=[0.0, -1.5, 1e3, 3.14159] + [0.01 * i for i in range(28)])])
@pytest.mark.parametrize("transposed", [False, True])
def test_scalings(spec, transposed, dtype):
    _run("paper", dtype, 65, spec=spec, transposed=transposed, positions=[i * i * 29 - 100 for i in range(65)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_and_negative_positions(dtype):
    far = [0, 1, -1, 2 ** 20 + 1, 2 ** 30, 2 ** 31 - 1, -2 ** 31, 123456789, -987654321]
    # an angle's fraction of a turn is exact to 2^-33: a frequency of 64 bits times a position of 31
    for layout in ("half", "interleaved"):
        _run("1b", dtype, len(far), layout=layout, positions=far)
        _run("odd", dtype, len(far), layout=layout, positions=far)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["1b", "paper", "odd"])
@pytest.mark.parametrize("kw", [dict(pad=64), dict(pad=5), dict(offset=1), dict(offset=8, pad=8), dict(out_pad=8), dict(out_pad=3), dict(in_place=True),
                                dict(in_place=True, pad=16), dict(sides="q"), dict(sides="k"), dict(magnitude=1.25)])
def test_strides_alignment_sides(kw, name, dtype):
    for layout in ("half", "interleaved"):
        for part in (None, 16):
            _run(name, dtype, 33, layout=layout, part=part, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_many_tokens(layout, dtype):
    _run("paper", dtype, 9001, layout=layout, spec=BANDS)
    _run("1b", dtype, 4000, layout=layout, part=64, pad=512)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_transposed_is_the_gradient(layout):
    """sum(w . R x) = sum(x . R^T w), and finite differences of it: the rotation is linear, so a difference of any size will do."""
    cfg = R.config("paper", "f32")
    rot = B.make_rotation(cfg, layout=layout, rotary_dim=32, magnitude=1.3, **BANDS)
    gen = R.generator(5)
    n = 40
    x, w, dx = (R.rows(gen, n, 320, "f32") for _ in range(3))
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 91

    def turn(v, back):
        out = torch.empty_like(v)
        B.gta_qk_rope(cfg, rot, v, 320, None, 0, pos, n, back, out, 320, None, 0)
        return out.double()

    grad = turn(w, True)
    lhs = (w.double() * (turn(x + dx, False) - turn(x, False))).sum(dim=1)
    rhs = (dx.double() * grad).sum(dim=1)
    # 320 products of terms of a few units, each with a handful of fp32 roundings
    assert torch.allclose(lhs, rhs, atol=320 * 16 * 2.0 ** -24 * 4, rtol=0)
    back = turn(turn(x, False).float(), True) / 1.3 ** 2
    assert torch.allclose(back[:, :32], x.double()[:, :32], atol=1e-5)


def test_nothing_to_do_and_current_stream():
    cfg = R.config("paper", "bf16")
    rot = B.make_rotation(cfg)
    x = torch.randn(8, 320, device="cuda").bfloat16()
    y = torch.full_like(x, 7.0)
    B.gta_qk_rope(cfg, rot, x, 320, None, 0, None, 0, False, y, 320, None, 0)
    torch.cuda.synchronize()
    assert bool((y == 7).all())
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        z = torch.empty_like(x)
        B.gta_qk_rope(cfg, rot, x, 320, None, 0, None, 8, False, z, 320, None, 0)
    s.synchronize()
    B.gta_qk_rope(cfg, rot, x, 320, None, 0, None, 8, False, y, 320, None, 0)
    assert torch.equal(y, z)
