"""gta_prefix_decode_attention against its formula in float64: prefixes and rows of every length, pages, rules, what must not leak."""
import random

import pytest
import torch

import rules_util as R
from paper_2506_17286_amd import binding as B

pytestmark = pytest.mark.gpu


class Cache:
    """Slots of random rows, contiguous or in shuffled pages; rows behind a slot's length hold `fill`."""

    def __init__(self, name, dtype, lens, room, gen, page=0, fill=float("nan"), seed=0, lens_tensor=None):
        sh = R.SHAPES.get(name, R.ROWS.get(name))
        self.lens, self.room = lens, room
        self.k, self.c = (torch.full((len(lens), room, w), fill, dtype=R.DT[dtype], device="cuda")
                          for w in (sh["n_kgroups"] * sh["head_dim"], sh["n_cgroups"] * sh["latent_dim"]))
        for i, n in enumerate(lens):
            n = min(max(n, 0), room)
            if n:
                self.k[i, :n], self.c[i, :n] = R.rows(gen, n, self.k.shape[2], dtype), R.rows(gen, n, self.c.shape[2], dtype)
        self.seq_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.status = torch.zeros_like(self.seq_lens)
        if page:
            pps = room // page
            order = torch.randperm(len(lens) * pps + 3, generator=torch.Generator().manual_seed(seed))[:len(lens) * pps]
            self.table = order.to(torch.int32).view(len(lens), pps).cuda()
            self.pools = [torch.full((len(lens) * pps + 3, page, t.shape[2]), fill, dtype=t.dtype, device="cuda") for t in (self.k, self.c)]
            for pool, t in zip(self.pools, (self.k, self.c)):
                pool[self.table.long().flatten()] = t.view(-1, page, t.shape[2])
            self.struct = B.make_paged_cache(*self.pools, self.seq_lens, self.status, self.table)
        else:
            self.pools = [self.k, self.c]
            self.struct = B.make_cache(self.k, self.c, self.seq_lens, self.status)

    def rows(self, slot):
        n = min(max(int(self.lens[slot]), 0), self.room) if 0 <= slot < len(self.lens) else 0
        return (self.k[slot, :n].double(), self.c[slot, :n].double()) if n else (self.k[0, :0].double(), self.c[0, :0].double())


def reference(cfg, q, prefix, prefix_slot, own, slots, rules):
    out = []
    pk, pc = prefix.rows(prefix_slot)
    for b in range(q.shape[0]):
        ok, oc = own.rows(slots[b])
        k, c = torch.cat([pk, ok]), torch.cat([pc, oc])
        n = k.shape[0]
        pos = torch.tensor([n - 1], device="cuda")
        lo = torch.tensor([rules["first"][b] if rules.get("first") else 0], device="cuda")
        hi = torch.tensor([rules["last"][b] if rules.get("last") else n - 1], device="cuda")
        out.append((R.attend(cfg, q[b:b + 1].double(), k, c, pos, lo, hi, rules.get("cap", 0.0), rules.get("slopes")), n))
    return out


def run(name, dtype, prefix_len, lens, *, page=0, prefix_page=None, cap=0.0, bias=False, first=None, last=None, slots=None, seed=0,
        prefix_room=None, room=None, prefix_slot=0, edit=None, scale=2.0, batch=None):
    cfg, sh, dt = R.config(name, dtype), R.SHAPES.get(name, R.ROWS.get(name)), R.DT[dtype]
    gen = R.generator(seed)
    unit = max(page, 64)
    prefix_page = page if prefix_page is None else prefix_page
    prefix = Cache(name, dtype, [3] * prefix_slot + [prefix_len], prefix_room or (max(prefix_len, 3) + unit) // unit * unit, gen, prefix_page, seed=seed + 1)
    own = Cache(name, dtype, lens, room or (max(max(lens), 0) + unit) // unit * unit, gen, page, seed=seed + 2)
    batch = batch or len(slots or lens)
    use = slots if slots is not None else list(range(batch))
    q = R.rows(gen, batch, sh["n_qgroups"] * sh["head_dim"], dtype, scale)
    slopes = torch.exp2(-8.0 * torch.arange(1, sh["n_qgroups"] + 1, device="cuda") / sh["n_qgroups"]) if bias else None
    rules = dict(cap=cap, slopes=slopes, first=first, last=last)
    if edit:
        edit(prefix, own, q)
    to = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")
    struct = B.make_score_rules(cap=cap, slopes=slopes, first=to(first), last=to(last)) if cap or bias or first or last else None
    out = torch.full((batch, sh["n_qgroups"] * sh["latent_dim"]), 55.0, dtype=dt, device="cuda")
    ws = B.alloc_workspace(B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFIX_DECODE, batch, prefix.room, own.room))
    B.gta_prefix_decode_attention(cfg, q, prefix.struct, prefix_slot, own.struct, to(slots), batch, struct, out, ws)
    torch.cuda.synchronize()
    for b, (ref, n) in enumerate(reference(cfg, q, prefix, prefix_slot, own, use, rules)):
        R.check(cfg, dtype, out[b:b + 1], *ref, n, f"{name} {dtype} prefix {prefix_len}, sequence {b} of {lens[use[b]] if 0 <= use[b] < len(lens) else None}")
    assert not bool(own.status.any()) and not bool(prefix.status.any())
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", sorted(R.SHAPES))
def test_layers(name, dtype):
    run(name, dtype, 150, [1, 70, 0, 33], seed=1)
    run(name, dtype, 333, [5, 200], cap=10.0, bias=True, page=16, seed=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", sorted(R.ROWS))
def test_layers_of_other_kernels(name, dtype):
    run(name, dtype, 40, [1, 75, 0, 200], seed=20, cap=8.0)
    run(name, dtype, 9300, [30, 130] * 10, bias=True, page=16, seed=21, first=[0, 9280] * 10)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix_len", [0, 1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 1000])
@pytest.mark.parametrize("name", ["paper", "1b"])
def test_lengths(name, prefix_len, dtype):
    run(name, dtype, prefix_len, [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 300], seed=prefix_len)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch", [1, 2, 6, 7, 8, 25, 26, 31, 32, 33, 64, 65, 130, 300])
@pytest.mark.parametrize("name", ["paper", "1b", "c2"])
def test_batches(name, batch, dtype):
    rng = random.Random(batch)
    run(name, dtype, 200, [rng.randint(0, 90) for _ in range(batch)], seed=batch, bias=batch % 2 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,prefix_page", [(16, 16), (64, 64), (256, 256), (16, 0), (0, 32), (24, 24), (5, 64), (8, 8)])
@pytest.mark.parametrize("name", ["paper", "1b", "wide"])
def test_pages(name, page, prefix_page, dtype):
    lens = [100, 3, 0, 64, 161]
    unit = max(page, 1)
    run(name, dtype, 190, lens, page=page, prefix_page=prefix_page, room=(200 + unit) // unit * unit,
        prefix_room=(256 + max(prefix_page, 1)) // max(prefix_page, 1) * max(prefix_page, 1), cap=30.0, seed=page + prefix_page)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["paper", "1b", "odd"])
def test_intervals(name, dtype):
    p, lens = 140, [50, 50, 50, 50, 0, 0, 20, 1, 50]
    first = [0, p, p + 10, p + 50, 0, p, 200, -7, 60]
    last = [R.INT_MAX, R.INT_MAX, p + 20, R.INT_MAX, R.INT_MAX, R.INT_MAX, 300, p, 50]
    run(name, dtype, p, lens, first=first, seed=3)
    run(name, dtype, p, lens, last=[139, 140, 0, -1, 500, 3, R.INT_MAX, 31, 32], seed=4, bias=True)
    run(name, dtype, p, lens, first=first, last=last, cap=20.0, bias=True, seed=5, page=16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slots_and_lengths_out_of_range(dtype):
    for name in ("paper", "1b", "odd"):
        run(name, dtype, 77, [10, 20, 30], slots=[2, 0, -1, 3, 1, 2], seed=6)
        run(name, dtype, 77, [-4, 20, 500], room=64, seed=7)
        run(name, dtype, 500, [4, 20], prefix_room=128, seed=8)
        run(name, dtype, -3, [4, 0], prefix_room=128, seed=9)
        run(name, dtype, 90, [4, 20], prefix_slot=2, seed=10)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefix_in_the_same_cache(dtype):
    cfg, sh = R.config("1b", dtype), R.SHAPES["1b"]
    gen = R.generator(11)
    both = Cache("1b", dtype, [130, 20, 64, 1], 192, gen, 16)
    q = R.rows(gen, 3, 512, dtype, 2.0)
    out = torch.empty((3, 2048), dtype=R.DT[dtype], device="cuda")
    ws = B.alloc_workspace(B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFIX_DECODE, 3, 192, 192))
    slots = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    B.gta_prefix_decode_attention(cfg, q, both.struct, 0, both.struct, slots, 3, None, out, ws)
    for b, (ref, n) in enumerate(reference(cfg, q, both, 0, both, [1, 2, 3], {})):
        R.check(cfg, dtype, out[b:b + 1], *ref, n, f"sequence {b}")


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["paper", "1b", "odd"])
def test_what_is_not_seen_does_not_leak(name, dtype, value):
    def edit(prefix, own, q):
        for t, slot, at in ((prefix, 0, 40), (prefix, 0, 99), (own, 0, 7), (own, 1, 20), (own, 3, 0)):
            t.c[slot, at, ::3] = value
            t.k[slot, at, 1] = float("nan")
        for t in (prefix, own):
            if t.pools[0] is not t.k:
                for pool, rows in zip(t.pools, (t.k, t.c)):
                    pool[t.table.long().flatten()] = rows.view(-1, pool.shape[1], rows.shape[2])
    first = [0, 41, 100, 120, 130, 90]
    last = [39, 98, R.INT_MAX, 129, R.INT_MAX, 98]
    for page in (0, 16):
        run(name, dtype, 120, [30, 30, 30, 30, 30, 30], first=first, last=last, edit=edit, seed=12, page=page)


@pytest.mark.parametrize("where", ["prefix", "own"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["paper", "1b", "wide", "odd"])
def test_an_infinite_latent_of_next_to_no_weight_shows(name, dtype, where):
    """One row has all the weight that fp32 can hold next to it; what is seen and not finite must not be lost with the rest."""
    cfg, sh, gen = R.config(name, dtype), R.SHAPES[name], R.generator(21)
    prefix, own = Cache(name, dtype, [600], 640, gen), Cache(name, dtype, [300, 40], 320, gen)
    dh = sh["head_dim"]
    for t in (prefix, own):   # q . k / sqrt(d_h): 160 nats below
        t.k.copy_(torch.full_like(t.k, -80.0 / dh ** 0.5))
    prefix.k[0, 3] = 80.0 / dh ** 0.5
    rows = prefix.c[0, 3].double().clone()
    (prefix if where == "prefix" else own).c[0, 200, 5] = float("inf")
    q = torch.ones(2, sh["n_qgroups"] * dh, dtype=R.DT[dtype], device="cuda")
    out = torch.zeros(2, sh["n_qgroups"] * sh["latent_dim"], dtype=R.DT[dtype], device="cuda")
    ws = B.alloc_workspace(B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFIX_DECODE, 2, prefix.room, own.room))
    B.gta_prefix_decode_attention(cfg, q, prefix.struct, 0, own.struct, None, 2, None, out, ws)
    qpc = sh["n_qgroups"] // sh["n_cgroups"]
    for b in range(2):
        for g in range(sh["n_qgroups"]):
            row, latent = out[b].view(-1, sh["latent_dim"])[g].double(), rows.view(-1, sh["latent_dim"])[g // qpc]
            hit = torch.zeros_like(row, dtype=torch.bool)
            hit[5] = g // qpc == 0 and (where == "prefix" or b == 0)
            assert not bool(torch.isfinite(row[hit]).any()), (b, g)
            assert bool((row[~hit] == latent[~hit]).all()), (b, g)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_query_that_is_not_finite_reaches_its_own_row_only(dtype):
    def edit(prefix, own, q):
        q[1] = float("nan")
        q[4, :70] = float("inf")
    for name in ("paper", "1b"):
        run(name, dtype, 100, [30, 40, 0, 9, 12], edit=edit, seed=13, cap=20.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["paper", "1b", "wide"])
def test_long_contexts(name, dtype):
    run(name, dtype, 9000, [20, 700, 3000], seed=14, cap=30.0)
    run(name, dtype, 3, [5000, 1, 2500, 0], seed=15, page=64)
    run(name, dtype, 5000, [1], seed=16, bias=True)


@pytest.mark.parametrize("cap,bias", [(0.0, False), (6.0, False), (0.0, True), (6.0, True)])
@pytest.mark.parametrize("name,batch", [("wide", 40), ("wide", 3), ("1b", 40), ("1b", 100), ("paper", 40)])
def test_many_readers_of_a_long_prefix(name, batch, cap, bias):
    run(name, "bf16", 8500, [(7 * i) % 50 for i in range(batch)], seed=30, cap=cap, bias=bias, page=32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_that_rise_and_fall(dtype):
    for sign in (1.0, -1.0):
        def edit(prefix, own, q):
            q.copy_(q.abs())
            for t in (prefix, own):
                for i, n in enumerate(t.lens):
                    t.k[i, :n] = (t.k[i, :n].abs() * sign * torch.linspace(0.0, 8.0, n, device="cuda")[:, None]).to(t.k.dtype)
        for name in ("paper", "1b"):
            run(name, dtype, 600, [300, 50], edit=edit, seed=17)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_latents(dtype):
    def edit(prefix, own, q):
        prefix.c.mul_(1e30)
        own.c.mul_(1e30)
    for name in ("paper", "1b"):
        run(name, dtype, 300, [100, 5], edit=edit, seed=18)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["paper", "1b"])
def test_captured_calls(name, dtype):
    """Two captured calls that share a workspace, replayed while both caches grow, between eager calls with it."""
    cfg, sh = R.config(name, dtype), R.SHAPES[name]
    gen = R.generator(19)
    prefix, own = Cache(name, dtype, [512], 512, gen), Cache(name, dtype, [256] * 20, 256, gen, 16)
    batches = (20, 7)
    qs = [R.rows(gen, b, sh["n_qgroups"] * sh["head_dim"], dtype, 2.0) for b in batches]
    ws = B.alloc_workspace(max(B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFIX_DECODE, b, 512, 256) for b in batches))
    rules = B.make_score_rules(cap=15.0)

    def fresh(i):
        return torch.full((batches[i], sh["n_qgroups"] * sh["latent_dim"]), 5.0, dtype=R.DT[dtype], device="cuda")

    def call(i, out):
        B.gta_prefix_decode_attention(cfg, qs[i], prefix.struct, 0, own.struct, None, batches[i], rules, out, ws)
        return out
    for i in range(2):
        call(i, fresh(i))
    torch.cuda.synchronize()
    outs, graphs = [fresh(0), fresh(1)], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i, outs[i])
        graphs.append(g)
    for step in range(5):
        prefix.seq_lens.fill_([0, 17, 512, 300, 1][step])
        own.seq_lens.copy_(torch.arange(20, dtype=torch.int32) * 13 % (step * 50 + 1))
        eager = [call(i, fresh(i)) for i in range(2)]
        for i in (step % 2, 1 - step % 2):
            outs[i].fill_(-1.0)
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(outs[i], eager[i])
