"""The operators together, as a decode step uses them: projection, norm and rotation, append into the 8-bit cache, attention,
value decoder, output projection.  Each stage is held to float64 on what the stage before it left; the step is run again
from a HIP graph, and on another stream; prompts go in and conversations come back out."""
import numpy as np
import pytest
import torch

from paper_2506_17286_amd import binding as B

import mx_util as M

pytestmark = pytest.mark.gpu

LAYERS = {"paper": dict(M.shape(5, 1, 1, 64, 128, nh=20, H=1280)), "1b": dict(M.shape(4, 4, 1, 128, 512, nh=16, H=2048))}


class Step:
    """Everything a decode step of `batch` sequences keeps."""

    def __init__(self, name, lens, page, seed=0):
        sh = self.sh = LAYERS[name]
        self.batch, H, dh, dl = len(lens), sh["d_model"], sh["head_dim"], sh["latent_dim"]
        nq, nk, nc, nh = (sh[n] for n in ("n_qgroups", "n_kgroups", "n_cgroups", "n_heads"))
        g = torch.Generator().manual_seed(seed)
        def bf(*s, std=1.0):
            return (torch.randn(s, generator=g) * std).to("cuda", torch.bfloat16)
        self.w = {"wq": bf(H, nq * dh, std=0.02), "wk": bf(H, nk * dh, std=0.02), "wc": bf(H, nc * dl, std=0.02),
                  "wg": bf(H, nh * dh, std=0.02), "wp": bf(nh, dl, dh, std=0.02), "wo": bf(nh * dh, H, std=0.02)}
        self.weights = B.make_weights(self.w)
        self.gains = [1 + 0.1 * bf(dh), 1 + 0.1 * bf(dh)]
        self.plain, self.cfg = (B.make_config(dtype="bf16", rope=r, **sh) for r in (False, True))
        self.cache = M.MxCache(sh, self.batch, 512, page, seed=1).fill(lens, np.random.default_rng(seed + 1))
        e = lambda w: torch.empty((self.batch, w), dtype=torch.bfloat16, device="cuda")   # noqa: E731
        self.x = bf(self.batch, H)
        self.q, self.k, self.c, self.g = e(nq * dh), e(nk * dh), e(nc * dl), e(nh * dh)
        self.qn, self.kn, self.l, self.heads, self.out = e(nq * dh), e(nk * dh), e(nq * dl), e(nh * dh), e(H)
        self.cu = torch.arange(self.batch + 1, dtype=torch.int32, device="cuda")
        self.ws = B.alloc_workspace(max(B.gta_workspace_bytes(self.plain, B.GTA_MODE_PREFILL, self.batch, self.batch, 1),
                                        B.gta_workspace_bytes(self.cfg, B.GTA_MODE_MX_DECODE, self.batch, 0, 512)))

    def run(self, stream=None):
        b, st = self.batch, stream
        B.gta_prefill_projection(self.plain, self.weights, self.x, None, b, b, 1, self.q, self.k, self.c, self.g, self.ws, stream=st)
        B.gta_qk_norm_rope(self.cfg, self.q, self.q.stride(0), self.k, self.k.stride(0), *self.gains, 1e-6, self.cache.seq_lens, b,
                           self.qn, self.kn, stream=st)
        B.gta_mx_cache_append(self.cfg, self.cache.struct, None, self.kn, self.kn.stride(0), self.c, self.c.stride(0), self.cu, b, 1, stream=st)
        B.gta_mx_decode_attention(self.cfg, self.qn, self.cache.struct, None, b, 0, self.l, self.ws, stream=st)
        B.gta_prefill_decoder(self.cfg, self.weights, self.l, self.g, b, self.heads, stream=st)
        B.gta_output_projection(self.cfg, self.weights, self.heads, b, self.out, stream=st)


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("name,page", [("paper", 0), ("paper", 16), ("1b", 64), ("1b", 0)])
def test_decode_steps(name, page):
    lens = [0, 1, 31, 200, 64, 333]
    s = Step(name, lens, page)
    sh, dh, dl = s.sh, s.sh["head_dim"], s.sh["latent_dim"]
    for _ in range(2):
        before = s.cache.seq_lens.cpu().numpy()
        s.run()
        torch.cuda.synchronize()
        assert (s.cache.seq_lens.cpu().numpy() == before + 1).all() and not s.cache.status.any()
        # norm and rotation of the projected rows
        for got, src, gain in ((s.qn, s.q, s.gains[0]), (s.kn, s.k, s.gains[1])):
            ref, mag = M.norm_rope(f64(src), f64(gain), 1e-6, before, dh, 10000.0, True)
            err = 32 * 2.0 ** -24 * mag
            assert (np.abs(f64(got) - ref) <= err + 2.0 ** -8 * (np.abs(ref) + err)).all()
        host = s.cache.host()
        for b in range(s.batch):
            at = s.cache.rows(b, 0, before[b] + 1)
            for i, src in ((0, s.kn), (1, s.c)):
                q, sc = M.quantise(f64(src)[b:b + 1])
                np.testing.assert_array_equal(M.E4M3[host[i][at[-1:]]], q)
                np.testing.assert_array_equal(host[i + 2][at[-1:]], sc)
            ref, mag, big = M.attention(sh, f64(s.qn)[b], M.values(host[0][at], host[2][at]), M.values(host[1][at], host[3][at]))
            assert (np.abs(f64(s.l)[b] - ref) <= M.attention_bound("bf16", sh, len(at), ref, mag, big)).all()
        # the decoder and the output projection, which are the framework's own, on the attention's output
        nh, nq = sh["n_heads"], sh["n_qgroups"]
        l, wp, gate = f64(s.l).reshape(s.batch, nq, dl), f64(s.w["wp"]), 1 / (1 + np.exp(-f64(s.g)))
        heads = np.concatenate([l[:, i * nq // nh] @ wp[i] for i in range(nh)], axis=1) * gate
        out = f64(s.heads) @ f64(s.w["wo"])
        for got, ref in ((f64(s.heads), heads), (f64(s.out), out)):
            assert np.linalg.norm(got - ref) <= 5e-3 * np.linalg.norm(ref)


@pytest.mark.parametrize("name,page", [("paper", 16), ("1b", 64)])
def test_step_replays_from_a_graph(name, page):
    lens = [0, 5, 130, 47]
    eager, graphed = Step(name, lens, page), Step(name, lens, page)
    warm = Step(name, lens, page)
    warm.run()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            graphed.run(stream=side)
    torch.cuda.synchronize()
    assert graphed.cache.seq_lens.cpu().tolist() == lens   # capturing ran nothing
    g = torch.Generator().manual_seed(9)
    for step in range(4):
        x = torch.randn(eager.x.shape, generator=g).to("cuda", torch.bfloat16)
        eager.x.copy_(x)
        graphed.x.copy_(x)
        graph.replay()
        eager.run()
        torch.cuda.synchronize()
        assert torch.equal(eager.out, graphed.out) and torch.equal(eager.l, graphed.l), f"replay {step}"
        for a, b in zip(eager.cache.host(), graphed.cache.host()):
            assert np.array_equal(a, b)
        assert graphed.cache.seq_lens.cpu().tolist() == [n + step + 1 for n in lens]
        _ = (eager.out.float() @ eager.out.float().t()).sum().item()


def test_two_streams_at_once():
    """Two batches with caches and workspaces of their own, each on its own stream, give what each gives alone."""
    alone = [Step("1b", [100, 7, 300], 16, seed=i) for i in range(2)]
    both = [Step("1b", [100, 7, 300], 16, seed=i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for s in alone:
            s.run()
            torch.cuda.synchronize()
        for s, st in zip(both, streams):
            s.run(stream=st)
        torch.cuda.synchronize()
        for a, b in zip(alone, both):
            assert torch.equal(a.out, b.out)


def test_prompt_in_and_conversation_out():
    """A ragged prompt batch: projected, normed and rotated, attended over as it is, stored in 8 bits; then its rows go back
    into a 16-bit cache with gta_cache_append and a chunk is run behind them."""
    sh = LAYERS["1b"]
    lens = [70, 1, 128]
    cu_np, total, H, dh = np.concatenate([[0], np.cumsum(lens)]), sum(lens), sh["d_model"], sh["head_dim"]
    s = Step("1b", [0, 0, 0], 16)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    x = torch.randn((total, H), generator=torch.Generator().manual_seed(3)).to("cuda", torch.bfloat16)
    cu = torch.tensor(cu_np, dtype=torch.int32, device="cuda")
    pos = torch.tensor(np.concatenate([np.arange(n) for n in lens]), dtype=torch.int32, device="cuda")
    q, k, c, gate = (torch.empty((total, w), **bf) for w in (512, 512, 512, 2048))
    qn, kn, l = (torch.empty((total, w), **bf) for w in (512, 512, 2048))
    ws = B.alloc_workspace(B.gta_workspace_bytes(s.plain, B.GTA_MODE_PREFILL, 3, total, max(lens)))
    B.gta_prefill_projection(s.plain, s.weights, x, cu, 3, total, max(lens), q, k, c, gate, ws)
    B.gta_qk_norm_rope(s.cfg, q, 512, k, 512, *s.gains, 1e-6, pos, total, qn, kn)
    B.gta_prefill_attention(s.cfg, qn, kn, c, cu, 3, total, max(lens), l)
    B.gta_mx_cache_append(s.cfg, s.cache.struct, None, kn, 512, c, 512, cu, 3, max(lens))
    assert s.cache.seq_lens.cpu().tolist() == lens
    kr, cr = (torch.empty((total, 512), **bf) for _ in range(2))
    B.gta_mx_cache_read(s.cfg, s.cache.struct, None, None, cu, 3, max(lens), kr, cr)
    for got, src in ((kr, kn), (cr, c)):
        v, sc = M.quantise(f64(src))
        np.testing.assert_array_equal(f64(got), v * np.repeat(2.0 ** (sc.astype(float) - 127), 32, axis=1))
    # the prompt's attention over exact rows and a query over the stored ones differ by the rows' rounding alone: the last
    # token's query over the stored rows is what attention over the rows read back gives
    last = torch.tensor(cu_np[1:] - 1, device="cuda")
    B.gta_mx_decode_attention(s.cfg, qn[last].contiguous(), s.cache.struct, None, 3, 0, s.l, s.ws)
    for b in range(3):
        rows = slice(cu_np[b], cu_np[b + 1])
        ref, mag, big = M.attention(sh, f64(qn)[cu_np[b + 1] - 1], f64(kr)[rows], f64(cr)[rows])
        assert (np.abs(f64(s.l)[b] - ref) <= M.attention_bound("bf16", sh, lens[b], ref, mag, big)).all()
    # back into 16 bits, and a chunk of new tokens behind them (queries and keys of the chunk as the projection gives them)
    k16, c16 = (torch.zeros((3, 256, 512), **bf) for _ in range(2))
    seq, st = (torch.zeros(3, dtype=torch.int32, device="cuda") for _ in range(2))
    cache16 = B.make_cache(k16, c16, seq, st)
    B.gta_cache_append(s.cfg, cache16, None, kr, cr, cu, 3, max(lens))
    xn = torch.randn((30, H), generator=torch.Generator().manual_seed(4)).to("cuda", torch.bfloat16)
    out = torch.empty((30, H), **bf)
    ws2 = B.alloc_workspace(B.gta_workspace_bytes(s.cfg, B.GTA_MODE_PREFILL_CHUNK, 3, 30, 10))
    B.gta_prefill_chunk(s.cfg, s.weights, xn, None, 3, 30, 10, cache16, None, out, ws2)
    assert seq.cpu().tolist() == [n + 10 for n in lens] and torch.isfinite(out).all()
    for b, n in enumerate(lens):
        assert torch.equal(k16[b, :n], kr[cu_np[b]:cu_np[b + 1]]) and torch.equal(c16[b, :n], cr[cu_np[b]:cu_np[b + 1]])


def test_tensors_that_are_not_on_the_device_are_refused():
    s = Step("paper", [3, 0], 0)
    s.run()
    host = torch.zeros_like(s.q, device="cpu")
    with pytest.raises(ValueError):
        B.gta_qk_norm_rope(s.cfg, host, s.q.stride(0), s.k, s.k.stride(0), None, None, 1e-6, None, 2, s.qn, s.kn)
    with pytest.raises(ValueError):
        B.gta_mx_cache_append(s.cfg, s.cache.struct, None, s.kn, 64, s.c, 128, s.cu.cpu(), 2, 1)
    with pytest.raises(ValueError):
        B.gta_mx_cache_read(s.cfg, s.cache.struct, None, None, s.cu, 2, 1, s.kn, s.c.cpu())
    with pytest.raises(ValueError):
        B.gta_mx_decode_attention(s.cfg, s.qn, s.cache.struct, None, 2, 0, s.l, s.ws.cpu())
    s.run()
    torch.cuda.synchronize()
