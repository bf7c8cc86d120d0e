"""gta_prefill_masked_attention against its formula in float64: caps, distances, intervals, lengths, strides, what must not leak."""
import random

import pytest
import torch

import rules_util as R
from paper_2506_17286_amd import binding as B

pytestmark = pytest.mark.gpu


def intervals(kind, n, rng):
    """First and last key of every token of a sequence of n."""
    lo, hi = [0] * n, list(range(n))
    if n == 0:
        return lo, hi
    if kind == "documents":
        at = 0
        while at < n:
            end = min(n, at + rng.randint(1, max(1, n // 2)))
            lo[at:end] = [at] * (end - at)
            at = end
    elif kind == "prefix":
        seen = rng.randint(0, n)
        hi = [max(i, seen - 1) for i in range(n)]
    elif kind == "window":
        w = rng.randint(1, n)
        lo = [max(0, i - w + 1) for i in range(n)]
    elif kind == "whole":
        lo, hi = [-5] * n, [R.INT_MAX] * n
    elif kind == "holes":        # some see nothing, in runs and alone
        for i in range(n):
            if rng.random() < 0.2 or (n > 40 and 7 <= i < 40):
                lo[i], hi[i] = rng.choice([(i + 1, i), (n, R.INT_MAX), (0, -1), (R.INT_MAX, -2 ** 31)])
    elif kind == "nothing":
        lo, hi = [1] * n, [0] * n
    elif kind == "any":          # nothing in order
        for i in range(n):
            a, b = rng.randint(-3, n + 2), rng.randint(-3, n + 2)
            lo[i], hi[i] = min(a, b), max(a, b)
    elif kind == "one":
        lo = hi = [rng.randrange(n) for _ in range(n)]
    return lo, hi


def slopes_of(nq):
    return torch.exp2(-8.0 * torch.arange(1, nq + 1, device="cuda") / nq)


def run(name, dtype, lens, kind="causal", cap=0.0, bias=False, seed=0, pads=None, offset=0, longest=None, equal=False, behind=0,
        scale=2.0, edit=None, ws=None, slopes=None, what=""):
    cfg, sh, dt = R.config(name, dtype), R.SHAPES[name], R.DT[dtype]
    rng, gen = random.Random(seed), R.generator(seed)
    total = sum(lens)
    widths = (sh["n_qgroups"] * sh["head_dim"], sh["n_kgroups"] * sh["head_dim"], sh["n_cgroups"] * sh["latent_dim"])
    x = []
    for i, w in enumerate(widths):
        pitch = w + (pads[i] if pads else 0)
        flat = R.rows(gen, 1, offset + (total + behind) * pitch, dtype, scale if i == 0 else 1.0)[0]
        x.append(flat[offset:].view(total + behind, pitch))
    q, k, c = (t[:, :w] for t, w in zip(x, widths))
    lo, hi = [], []
    for n in lens:
        a, b = intervals(kind, n, rng)
        lo += a
        hi += b
    lo, hi = lo + [0] * behind, hi + [R.INT_MAX] * behind
    first, last = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (lo, hi))
    if bias and slopes is None:
        slopes = slopes_of(sh["n_qgroups"])
    if edit:
        edit(q, k, c, lo, hi)
    plain = kind == "causal"
    rules = B.make_score_rules(cap=cap, slopes=slopes, first=None if plain else first, last=None if plain else last)
    cu = None if equal else torch.tensor([0] + lens, dtype=torch.int32, device="cuda").cumsum(0).to(torch.int32)
    longest = longest or max(lens)
    out = torch.full((total + behind, sh["n_qgroups"] * sh["latent_dim"]), 77.0, dtype=dt, device="cuda")
    if ws is None:
        ws = B.alloc_workspace(B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFILL_MASKED, len(lens), total + behind, longest))
    B.gta_prefill_masked_attention(cfg, q, q.stride(0), k, k.stride(0), c, c.stride(0), cu, len(lens), total + behind, longest,
                                   None if plain and not cap and not bias else rules, out, ws)
    torch.cuda.synchronize()
    at = 0
    for n in lens:
        rows = slice(at, at + n)
        own = torch.arange(n, device="cuda")
        ref = R.attend(cfg, q[rows].double(), k[rows].double(), c[rows].double(), own, first[rows].long(), last[rows].long().clamp(max=n - 1) if not plain else own,
                       cap, slopes)
        R.check(cfg, dtype, out[rows], *ref, n, f"{what} {name} {dtype} {kind} at {at}, {n} tokens")
        at += n
    assert bool((out[total:] == 77.0).all())
    return out


KINDS = ["causal", "documents", "prefix", "window", "whole", "holes", "nothing", "any", "one"]
LENS = [1, 33, 2, 150, 64, 31]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", ["paper", "1b", "c2", "odd"])
def test_masks(name, kind, dtype):
    run(name, dtype, LENS, kind, seed=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", sorted(R.SHAPES))
def test_layers(name, dtype):
    run(name, dtype, [70, 129, 1], "documents", cap=20.0, bias=True, seed=5)
    run(name, dtype, [257], "causal", seed=6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300])
def test_lengths(n, dtype):
    run("paper", dtype, [n], "any", seed=n)
    run("1b", dtype, [n, n], "causal", cap=5.0, equal=True, seed=n)
    run("l128", dtype, [n], "prefix", bias=True, seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [0.01, 1.0, 30.0, 1e6, 1e30])
@pytest.mark.parametrize("bias", [False, True])
def test_caps(cap, bias, dtype):
    run("paper", dtype, [97, 20], "whole", cap=cap, bias=bias, seed=8)
    run("1b", dtype, [97, 20], "window", cap=cap, bias=bias, seed=9, scale=20.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slopes_of_any_sign_and_size(dtype):
    for values in ([0.0, 0.0, 0.0, 0.0, 0.0], [50.0, 3.0, 1.0, -0.01, 0.5], [-1.0, -0.2, 1e-30, 700.0, 1e4]):
        run("paper", dtype, [300, 40], "causal", bias=True, slopes=torch.tensor(values, device="cuda"), seed=4)
        run("paper", dtype, [300, 40], "whole", bias=True, slopes=torch.tensor(values, device="cuda"), seed=4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["paper", "1b", "wide"])
@pytest.mark.parametrize("kind", ["causal", "documents", "window", "prefix"])
def test_long_sequences(name, kind, dtype):
    run(name, dtype, [1500 if name == "wide" else 2500, 700], kind, cap=30.0 if kind == "prefix" else 0.0, bias=kind == "window", seed=11)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences(dtype):
    rng = random.Random(2)
    run("paper768", dtype, [rng.randint(0, 60) for _ in range(300)] + [0, 5], "documents", seed=12)
    run("paper768", dtype, [0, 0, 3, 0], "holes", seed=12)
    run("l256", dtype, [rng.choice([1, 2, 200]) for _ in range(70)], "causal", bias=True, seed=13)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pads,offset", [((64, 64, 64), 0), ((8, 16, 24), 8), ((1, 0, 0), 0), ((0, 3, 0), 0), ((0, 0, 5), 0), ((8, 8, 8), 1), ((4, 4, 4), 4)])
def test_strides_and_alignment(pads, offset, dtype):
    for name in ("paper", "1b"):
        run(name, dtype, [40, 140], "documents", cap=10.0, pads=pads, offset=offset, seed=14)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_behind_the_last_sequence_and_loose_bounds(dtype):
    for name in ("paper", "1b", "odd"):
        run(name, dtype, [40, 0, 130], "causal", behind=9, longest=500, seed=15)
        run(name, dtype, [40, 0, 130], "whole", behind=200, longest=4000, seed=15)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["paper", "1b", "odd", "c2"])
def test_what_is_not_seen_does_not_leak(name, dtype, value):
    """Values that are not finite in keys and latents that some tokens of the same blocks do not see."""
    def edit(q, k, c, lo, hi):
        c[5] = value                 # seen by tokens of its document only, or from itself on
        c[70, 3] = value
        k[100, :7] = float("nan")
        c[100] = value
        if c.shape[0] > 130:
            c[130, ::2] = value
    for kind in ("causal", "documents", "window", "any", "holes"):
        run(name, dtype, [160, 30], kind, edit=edit, seed=16, what=str(value))
        # with a bound of more keys tiles are listed and their keys shared out
        run(name, dtype, [160, 30], kind, edit=edit, seed=16, what=str(value), longest=5000, cap=20.0, bias=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", ["paper", "1b", "c2", "q6k2c3", "l192"])
def test_masks_of_listed_and_cut_tiles(name, kind, dtype):
    run(name, dtype, LENS, kind, seed=23, longest=2000, bias=True)
    run(name, dtype, [1, 700, 0, 400], kind, seed=24, longest=3000)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_tiles_than_the_list_keeps(dtype):
    """More than four tiles a thread of the list's workgroup, and more sequences than its LDS has room for."""
    rng = random.Random(3)
    run("paper768", dtype, [rng.choice([0, 1, 2, 3]) for _ in range(4500)], "any", seed=25, longest=2000)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_scores_and_queries(dtype):
    def edit(q, k, c, lo, hi):
        q[9] = float("nan")
        q[40, :] = 0.0
        k[20, :] = torch.finfo(k.dtype).max / 4
        q[50, :] = 0.0
    run("paper", dtype, [120], "documents", cap=20.0, edit=edit, seed=17)

    def large(q, k, c, lo, hi):
        q.mul_(50.0)
        c.mul_(1e30)
    run("paper", dtype, [300], "causal", edit=large, seed=18)
    run("1b", dtype, [300], "prefix", edit=large, seed=18)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_that_rise_and_fall(dtype):
    """Maxima that move far, up and down, with every block of keys."""
    for sign in (1.0, -1.0):
        def edit(q, k, c, lo, hi):
            n = k.shape[0]
            q.copy_(q.abs())
            k.copy_((k.abs() * sign * torch.linspace(0.0, 6.0, n, device="cuda")[:, None]).to(k.dtype))
        run("paper", dtype, [400], "causal", edit=edit, seed=19)
        run("1b", dtype, [400], "whole", edit=edit, seed=19)
        run("1b", dtype, [400], "documents", cap=50.0, edit=edit, seed=19)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_result_twice_and_on_another_stream(dtype):
    a = run("1b", dtype, [600, 90], "documents", cap=30.0, bias=True, seed=20)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = run("1b", dtype, [600, 90], "documents", cap=30.0, bias=True, seed=20)
    assert torch.equal(a, b)


@pytest.mark.parametrize("name", ["paper", "1b"])
def test_without_rules_it_is_the_prefill_attention(name):
    cfg, sh = R.config(name, "bf16"), R.SHAPES[name]
    gen, n = R.generator(21), 500
    q, k, c = (R.rows(gen, n, w, "bf16") for w in (sh["n_qgroups"] * sh["head_dim"], sh["n_kgroups"] * sh["head_dim"], sh["n_cgroups"] * sh["latent_dim"]))
    a, b = (torch.empty((n, sh["n_qgroups"] * sh["latent_dim"]), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = B.alloc_workspace(B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFILL_MASKED, 2, n, 250))
    B.gta_prefill_masked_attention(cfg, q, q.stride(0), k, k.stride(0), c, c.stride(0), None, 2, n, 250, None, a, ws)
    B.gta_prefill_attention(cfg, q, k, c, None, 2, n, 250, b)
    # two results of the same formula, each within its bound: weights of 16 bits and a rounded result
    assert torch.allclose(a.float(), b.float(), atol=2 * 3 * 2.0 ** -8 * c.float().abs().max().item(), rtol=2.0 ** -7)
    assert (a.float() - b.float()).norm() <= 5e-3 * b.float().norm()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["paper", "1b"])
def test_captured_calls(name, dtype):
    """Two captured calls that share a workspace, replayed between eager calls of other lengths with it."""
    cfg, sh, dt = R.config(name, dtype), R.SHAPES[name], R.DT[dtype]
    gen, n = R.generator(22), 700
    q, k, c = (R.rows(gen, n, w, dtype, 2.0) for w in (sh["n_qgroups"] * sh["head_dim"], sh["n_kgroups"] * sh["head_dim"], sh["n_cgroups"] * sh["latent_dim"]))
    first = torch.zeros(n, dtype=torch.int32, device="cuda")
    rules = B.make_score_rules(cap=25.0, first=first)
    ws = B.alloc_workspace(B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFILL_MASKED, 2, n, n))
    cu = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 300, n], [0, 1, n])]

    def call(i, out):
        B.gta_prefill_masked_attention(cfg, q, q.stride(0), k, k.stride(0), c, c.stride(0), cu[i], 2, n, n, rules, out, ws)
        return out

    def fresh():
        return torch.full((n, sh["n_qgroups"] * sh["latent_dim"]), 5.0, dtype=dt, device="cuda")
    eager = [call(i, fresh()) for i in range(2)]
    torch.cuda.synchronize()
    graphs, outs = [], [fresh(), fresh()]
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i, outs[i])
        graphs.append(g)
    for step in range(4):
        first.fill_(step * 60)
        eager = [call(i, fresh()) for i in range(2)]
        for i in (step % 2, 1 - step % 2):
            outs[i].fill_(-1.0)
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(outs[i], eager[i])
