"""Attention with rules where one latent of one column is not finite, and keys are shared out over pieces: its column shows it to the
rows that see it, and no other column or row changes, whichever workgroup, wave or piece had it."""
import pytest
import torch

import rules_util as R
import test_gpu_masked_attention as M
import test_gpu_prefix_decode as P

pytestmark = pytest.mark.gpu


def rising(k, n):
    """Keys whose scores with queries of positive elements rise from the last one to the first by about 4 (5.8 in units of log 2), so that the
    maxima of blocks differ by less than what makes a kernel change what its weights refer to."""
    dh_ramp = 2.5 / 8.0 * torch.linspace(1.0, 0.0, n, device="cuda")[:, None]
    k[:n] = (0.3 * k[:n].float() + dh_ramp).to(k.dtype)


def columns(latent):
    """One in each block of 32 columns of the first 128, and in the first and last of every 64 behind them."""
    return [5, 37, 70, 127] if latent == 128 else [0, 70, latent // 2 - 1, latent // 2 + 3, latent - 1]


@pytest.fixture
def faint(monkeypatch):
    """Where a distance leaves an infinite latent a weight that 32 bits cannot hold, its product is 0 * inf = NaN there and inf in 64 bits:
    exp(-slope * distance) is below 2^-126, the least normal number, from slope * distance = 88 on, and the distances here go up to
    1790 with slopes of up to 1/2 (448 and more, 895 at most).  Such an element has to be not finite; what else is not, as elsewhere."""
    attend, check, found = R.attend, R.check, []

    def attend_noting(cfg, q, k, c, *rest):
        one = torch.zeros_like(c)
        one[~torch.isfinite(c).all(dim=1)] = 1.0
        found[:] = [attend(cfg, q, k, one, *rest)[0] < 2.0 ** -126]
        return attend(cfg, q, k, c, *rest)

    def check_noting(cfg, dtype, got, out, *rest):
        out, got = out.clone(), got.double()
        weak = found[0] & ~torch.isfinite(out)
        assert not bool(torch.isfinite(got[weak]).any())
        out[weak] = got[weak] = 0.0
        check(cfg, dtype, got, out, *rest)
    monkeypatch.setattr(R, "attend", attend_noting)
    monkeypatch.setattr(R, "check", check_noting)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["paper", "1b", "wide", "l256", "l192", "q8k4c2"])
@pytest.mark.parametrize("ramp", [False, True])
def test_prompts(faint, name, dtype, value, ramp):
    latent = R.SHAPES[name]["latent_dim"]
    n = 1800
    for i, col in enumerate(columns(latent)):
        def edit(q, k, c, lo, hi):
            if ramp:
                q.copy_(q.abs())
                rising(k, n)
            c[[n - 10, 9][i % 2], col] = value
        M.run(name, dtype, [n], "causal", edit=edit, seed=31 + i, what=f"{value} in column {col}", bias=i % 2 == 1)
        M.run(name, dtype, [70, 200, 33], "documents", edit=lambda q, k, c, lo, hi: c[100, col].fill_(value), seed=41 + i, longest=3000,
              what=f"{value} in column {col}")


@pytest.mark.parametrize("value", [float("nan"), float("-inf")])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name,batch", [("paper", 2), ("paper", 9), ("1b", 3), ("1b", 40), ("1b", 70), ("wide", 3), ("wide", 40), ("l256", 5), ("l128", 4),
                                        ("l192", 4), ("c2", 3)])
@pytest.mark.parametrize("ramp", [False, True])
def test_prefixes(name, batch, dtype, value, ramp):
    latent = R.SHAPES[name]["latent_dim"]
    for i, col in enumerate(columns(latent)):
        first = [[0, 500, 1200][b % 3] for b in range(batch)]   # (some do not see the prefix's bad row, some nothing of the prefix)

        def edit(prefix, own, q):
            if ramp:
                q.copy_(q.abs())
                rising(prefix.k[0], 1200)
                for b in range(batch):
                    rising(own.k[b], own.lens[b])
            prefix.c[0, 480, col] = value
            own.c[1, 3, latent - 1 - col] = value
        P.run(name, dtype, 1200, [30 + 7 * (b % 11) for b in range(batch)], first=first, edit=edit, seed=51 + i, cap=0.0 if i % 2 else 30.0)
