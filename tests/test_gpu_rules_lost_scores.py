"""Keys whose products with a query pass fp32's range downwards: their weight is 0, and what they hold that is not finite shows in the rows that
see them, whether they are alone in a piece of the keys or not."""
import pytest
import torch

import rules_util as R
import test_gpu_masked_attention as M
import test_gpu_prefix_decode as P

pytestmark = pytest.mark.gpu


def lost(q, k, rows):
    """Scores of -infinity (in 64 bits: -1e59 and less) for `rows`, ordinary ones for the others."""
    q[:, ::2] = 0.0
    q[:, 1::2] = 1e30
    k[:, 1::2] = 0.0
    k[rows, 1::2] = -1e30
    q[:, 0] = 1.0
    if q.shape[1] > 128:
        q[:, 128] = 1.0


@pytest.mark.parametrize("value", [float("nan"), float("inf"), 1.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["paper", "1b", "wide", "l192", "odd"])
def test_prompts(name, dtype, value):
    for rows, bad in ((slice(0, 900), 500), (slice(1000, 2000), 1500), (slice(3, 40), 7)):
        def edit(q, k, c, lo, hi):
            lost(q, k, rows)
            c[bad, 5] = value
        M.run(name, dtype, [2000], "whole", edit=edit, seed=81, what=f"{rows} {value}")


@pytest.mark.parametrize("value", [float("nan"), float("inf"), 1.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name,batch", [("paper", 2), ("1b", 2), ("1b", 70), ("wide", 3), ("l192", 2), ("odd", 2)])
@pytest.mark.parametrize("where", ["prefix", "own"])
def test_prefixes(name, batch, dtype, value, where):
    def edit(prefix, own, q):
        if where == "prefix":
            lost(q, prefix.k[0], slice(0, 700))
            own.k[:, :, 1::2] = 0.0
            prefix.c[0, 500, 5] = value
        else:
            for i in range(batch):
                lost(q, own.k[i], slice(0, 900))
            prefix.k[:, :, 1::2] = 0.0
            own.c[0, 500, 5] = value
    lens = [1000] * batch
    P.run(name, dtype, 1500, lens, edit=edit, seed=82)
    P.run(name, dtype, 1500, lens, edit=edit, seed=83, first=[[0, 1100, 200][i % 3] for i in range(batch)])
