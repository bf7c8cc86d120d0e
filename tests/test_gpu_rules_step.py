"""The operators together, as a serving loop uses them: a system prompt goes in once, conversations behind it are prefilled and decoded
step by step, with rotary positions scaled for long contexts, capped scores and distances.  Each stage is held to float64 on what the
stage before it left; decode steps are compared with one attention over whole conversations; steps run again from a HIP graph and on
another stream."""
import numpy as np
import pytest
import torch

import rules_util as R
from paper_2506_17286_amd import binding as B

pytestmark = pytest.mark.gpu

LAYERS = {"paper": dict(R.SHAPES["paper"], d_model=1280, n_heads=20), "1b": dict(R.SHAPES["1b"], d_model=2048, n_heads=16)}
BANDS = dict(scaling="bands", factor=8.0, trained_len=64.0, slow_turns=1.0, fast_turns=4.0)


class Loop:
    """A layer, its caches and the buffers of prefills and decode steps."""

    def __init__(self, name, prefix_len, lens, page, layout, room=256, seed=0):
        sh = self.sh = LAYERS[name]
        H, dh, dl = sh["d_model"], sh["head_dim"], sh["latent_dim"]
        nq, nk, nc, nh = (sh[n] for n in ("n_qgroups", "n_kgroups", "n_cgroups", "n_heads"))
        self.gen, self.batch, self.lens, self.prefix_len, self.layout = R.generator(seed), len(lens), lens, prefix_len, layout
        self.cfg = B.make_config(dtype="bf16", rope=False, **sh)
        self.part = dh // 2
        self.rotation = B.make_rotation(self.cfg, layout=layout, rotary_dim=self.part, **BANDS)
        self.slopes = torch.exp2(-2.0 * torch.arange(1, nq + 1, device="cuda"))
        self.cap = 15.0
        self.widths = dict(q=nq * dh, k=nk * dh, c=nc * dl, g=nh * dh)
        w = {"wq": (H, nq * dh), "wk": (H, nk * dh), "wc": (H, nc * dl), "wg": (H, nh * dh), "wp": (nh, dl, dh)}
        self.w = {n: (torch.empty(s, device="cuda").normal_(0, 0.04, generator=self.gen)).bfloat16() for n, s in w.items()}
        self.weights = B.make_weights(self.w)
        self.prefix, self.prefix_seen = self.cache(1, (prefix_len + 63) // 64 * 64, page)
        self.own, _ = self.cache(self.batch, room, page)
        self.room = room

    def cache(self, slots, room, page):
        n = torch.zeros(slots, dtype=torch.int32, device="cuda")
        status = torch.zeros_like(n)
        shape = (slots * (room // page), page) if page else (slots, room)
        parts = [torch.zeros(shape + (self.widths[x],), dtype=torch.bfloat16, device="cuda") for x in "kc"]
        table = torch.randperm(shape[0], generator=torch.Generator().manual_seed(5)).int().view(slots, -1).cuda() if page else None
        struct = B.make_paged_cache(*parts, n, status, table) if page else B.make_cache(*parts, n, status)
        struct.keep = (parts, n, status, table)
        return struct, n

    def project(self, x, cu, batch, longest):
        t = x.shape[0]
        out = {n: torch.empty((t, w), dtype=torch.bfloat16, device="cuda") for n, w in self.widths.items()}
        ws = B.alloc_workspace(B.gta_workspace_bytes(self.cfg, B.GTA_MODE_PREFILL, batch, t, longest))
        B.gta_prefill_projection(self.cfg, self.weights, x, cu, batch, t, longest, *(out[n] for n in "qkcg"), ws)
        return out

    def turn(self, p, positions):
        """In place; checked against the rotation in extended precision."""
        before = {n: p[n].double().cpu().numpy() for n in "qk"}
        B.gta_qk_rope(self.cfg, self.rotation, p["q"], p["q"].stride(0), p["k"], p["k"].stride(0), positions, p["q"].shape[0], False,
                      p["q"], p["q"].stride(0), p["k"], p["k"].stride(0))
        dh = self.sh["head_dim"]
        freq = R.frequencies(self.part, **BANDS)
        for n in "qk":
            ref, size = R.rotate(before[n], p[n].shape[1] // dh, dh, self.part, freq, positions.cpu().numpy(), self.layout == "interleaved", False)
            tol = 2.0 ** -8 * np.abs(ref) + 4e-7 * size
            assert np.all(np.abs(p[n].double().cpu().numpy() - ref) <= tol)

    def x(self, n):
        return torch.empty((n, self.sh["d_model"]), device="cuda").normal_(0, 1, generator=self.gen).bfloat16()


@pytest.mark.parametrize("name,page,layout", [("paper", 16, "interleaved"), ("1b", 0, "half"), ("1b", 64, "interleaved")])
def test_a_serving_loop(name, page, layout):
    lens = [1, 40, 7, 100, 33]
    s = Loop(name, 130, lens, page, layout)
    cfg, P, b = s.cfg, s.prefix_len, s.batch
    cu1 = torch.tensor([0, P], dtype=torch.int32, device="cuda")
    # the system prompt, once
    pre = s.project(s.x(P), cu1, 1, P)
    s.turn(pre, torch.arange(P, dtype=torch.int32, device="cuda"))
    B.gta_cache_append(cfg, s.prefix, None, pre["k"], pre["c"], cu1, 1, P)
    # conversations behind it: their rows go into caches of their own
    cu = torch.tensor([0] + lens, dtype=torch.int32, device="cuda").cumsum(0).int()
    chat = s.project(s.x(sum(lens)), cu, b, max(lens))
    s.turn(chat, torch.cat([P + torch.arange(n, dtype=torch.int32, device="cuda") for n in lens]))
    B.gta_cache_append(cfg, s.own, None, chat["k"], chat["c"], cu, b, max(lens))
    whole = [{n: torch.cat([pre[n], chat[n][cu[i]:cu[i + 1]]]) for n in "qkc"} for i in range(b)]

    def attended(rows):
        """One attention over the conversations as they are by now, the system prompt in front of each; the prompt seen from everywhere."""
        ns = [r["q"].shape[0] for r in rows]
        q, k, c = (torch.cat([r[n] for r in rows]) for n in "qkc")
        last = torch.cat([torch.arange(n, device="cuda").clamp(min=P - 1) for n in ns]).int()
        rules = B.make_score_rules(cap=s.cap, slopes=s.slopes, last=last)
        ends = torch.tensor([0] + ns, dtype=torch.int32, device="cuda").cumsum(0).int()
        l = torch.empty((sum(ns), s.sh["n_qgroups"] * s.sh["latent_dim"]), dtype=torch.bfloat16, device="cuda")
        ws = B.alloc_workspace(B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFILL_MASKED, b, sum(ns), max(ns)))
        B.gta_prefill_masked_attention(cfg, q, q.stride(0), k, k.stride(0), c, c.stride(0), ends, b, sum(ns), max(ns), rules, l, ws)
        for i, n in enumerate(ns):
            at = slice(int(ends[i]), int(ends[i + 1]))
            ref = R.attend(cfg, q[at].double(), k[at].double(), c[at].double(), torch.arange(n, device="cuda"), torch.zeros(n, dtype=torch.long, device="cuda"),
                           last[at].long(), s.cap, s.slopes)
            R.check(cfg, "bf16", l[at], *ref, n, f"conversation {i}")
        return l, ends

    attended(whole)
    rules = B.make_score_rules(cap=s.cap, slopes=s.slopes)
    ws = B.alloc_workspace(B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFIX_DECODE, b, s.prefix.max_seq, s.room))
    own_lens = s.own.keep[1]
    one = torch.arange(b + 1, dtype=torch.int32, device="cuda")
    for step in range(3):
        new = s.project(s.x(b), None, b, 1)
        s.turn(new, own_lens + P)
        B.gta_cache_append(cfg, s.own, None, new["k"], new["c"], one, b, 1)
        l = torch.empty((b, s.sh["n_qgroups"] * s.sh["latent_dim"]), dtype=torch.bfloat16, device="cuda")
        B.gta_prefix_decode_attention(cfg, new["q"], s.prefix, 0, s.own, None, b, rules, l, ws)
        whole = [{n: torch.cat([whole[i][n], new[n][i:i + 1]]) for n in "qkc"} for i in range(b)]
        full, ends = attended(whole)
        for i in range(b):
            r = whole[i]
            n = r["q"].shape[0]
            ref = R.attend(cfg, r["q"][-1:].double(), r["k"].double(), r["c"].double(), torch.tensor([n - 1], device="cuda"), torch.tensor([0], device="cuda"),
                           torch.tensor([n - 1], device="cuda"), s.cap, s.slopes)
            R.check(cfg, "bf16", l[i:i + 1], *ref, n, f"step {step}, sequence {i}")
            R.check(cfg, "bf16", full[ends[i + 1] - 1:ends[i + 1]], *ref, n, f"step {step}, conversation {i}")
        heads = torch.empty((b, s.widths["g"]), dtype=torch.bfloat16, device="cuda")
        B.gta_prefill_decoder(cfg, s.weights, l, new["g"], b, heads)
        assert bool(torch.isfinite(heads).all())
    assert own_lens.tolist() == [n + 3 for n in lens] and not bool(s.own.keep[2].any())


@pytest.mark.parametrize("name", ["paper", "1b"])
def test_a_captured_decode_step(name):
    """Rotation, append and attention of a step in one graph, replayed while the caches grow, against eager steps and another stream."""
    lens = [3, 50, 0, 20]
    loops = [Loop(name, 200, lens, 16, "half", seed=3) for _ in range(3)]
    for s in loops:
        cu = torch.tensor([0, 200], dtype=torch.int32, device="cuda")
        ends = torch.tensor([0] + lens, dtype=torch.int32, device="cuda").cumsum(0).int()
        g = R.generator(9)
        B.gta_cache_append(s.cfg, s.prefix, None, R.rows(g, 200, s.widths["k"], "bf16"), R.rows(g, 200, s.widths["c"], "bf16"), cu, 1, 200)
        B.gta_cache_append(s.cfg, s.own, None, R.rows(g, sum(lens), s.widths["k"], "bf16"), R.rows(g, sum(lens), s.widths["c"], "bf16"), ends, 4, max(lens))
        s.one = torch.arange(5, dtype=torch.int32, device="cuda")
        s.rows = [torch.empty((4, s.widths[n]), dtype=torch.bfloat16, device="cuda") for n in "qkc"]
        s.l = torch.empty((4, s.sh["n_qgroups"] * s.sh["latent_dim"]), dtype=torch.bfloat16, device="cuda")
        s.ws = B.alloc_workspace(B.gta_workspace_bytes(s.cfg, B.GTA_MODE_PREFIX_DECODE, 4, s.prefix.max_seq, s.room))
        s.positions = torch.empty(4, dtype=torch.int32, device="cuda")
        s.rules = B.make_score_rules(cap=12.0)

    def step(s):
        q, k, c = s.rows
        torch.add(s.own.keep[1], 200, out=s.positions)
        B.gta_qk_rope(s.cfg, s.rotation, q, q.stride(0), k, k.stride(0), s.positions, 4, False, q, q.stride(0), k, k.stride(0))
        B.gta_cache_append(s.cfg, s.own, None, k, c, s.one, 4, 1)
        B.gta_prefix_decode_attention(s.cfg, q, s.prefix, 0, s.own, None, 4, s.rules, s.l, s.ws)

    def feed(s, n):
        g = R.generator(100 + n)
        for t in s.rows:
            t.copy_(R.rows(g, 4, t.shape[1], "bf16"))

    eager, captured, streamed = loops
    for s in loops:
        feed(s, 0)
        step(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    stream = torch.cuda.Stream()
    for n in range(1, 5):
        for s in loops:
            feed(s, n)
        torch.cuda.synchronize()
        graph.replay()
        step(eager)
        with torch.cuda.stream(stream):
            step(streamed)
        torch.cuda.synchronize()
        assert torch.equal(eager.l, captured.l) and torch.equal(eager.l, streamed.l)
        assert bool(torch.isfinite(eager.l).all())
        assert eager.own.keep[1].tolist() == captured.own.keep[1].tolist() == [v + n + 1 for v in lens]
