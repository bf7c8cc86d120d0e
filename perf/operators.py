"""The serving operators around a cache of 8-bit keys and latent values, as measurable cases.

One case is one pass through one operator on tensors that already live on the GPU:

  norm_rope  RMS norm of every query and key head, then its rotation, in one pass over the projected rows
  append     new key and latent rows are quantised into the cache behind each sequence's rows
  read       cached rows are read back in 16 or 32 bits
  attend     one new token per sequence attends over all its cached rows

A quantised row is stored in blocks of 32 elements: e4m3 codes, and one byte e + 127 a block, for the value code * 2^e.
e is the least exponent with which the block's largest finite magnitude is at most 448 * 2^e, kept within -117 .. 119.

With `own` false a pass is made of elementary torch operations in 32 bits (angles in 64), with `own` true of the
library's calls.  The layers:

  paper    one attention layer of the paper's GTA-1B model: 5 maps and one key of 64, one latent of 128
  paper768 the same family at width 768: 3 maps
  1b       4 maps and keys of 128, one latent of 512
  wide     8 maps and keys of 128, one latent of 1024
"""
from __future__ import annotations

import math
import random
from typing import Dict, List

import torch

own = False

LAYERS: Dict[str, Dict] = {
    "paper": dict(d_model=1280, n_heads=20, n_qgroups=5, n_kgroups=1, n_cgroups=1, head_dim=64, latent_dim=128),
    "paper768": dict(d_model=768, n_heads=12, n_qgroups=3, n_kgroups=1, n_cgroups=1, head_dim=64, latent_dim=128),
    "1b": dict(d_model=2048, n_heads=16, n_qgroups=4, n_kgroups=4, n_cgroups=1, head_dim=128, latent_dim=512),
    "wide": dict(d_model=4096, n_heads=32, n_qgroups=8, n_kgroups=8, n_cgroups=1, head_dim=128, latent_dim=1024),
}
ROPE_BASE = 10000.0
EPS = 1e-6
BLOCK = 32


def _case(kind: str, layer: str, dtype: str, batch: int, new: int, cached: int = 0, shortest: int = 0, page: int = 0,
          fused: bool = False, mix: int = 0) -> Dict:
    """new: rows of the longest sequence in this call (append, read, norm_rope; 1 for attend); cached: rows of the
    longest sequence before it; shortest > 0: lengths spread over [shortest, longest] by the generator `mix`; page:
    rows of a page, 0 for contiguous slots; fused: the rows are columns of one wide projection's output."""
    return dict(kind=kind, layer=layer, dtype=dtype, batch=batch, new=new, cached=cached, shortest=shortest, page=page,
                fused=fused, mix=mix)


def listed() -> List[Dict]:
    cases = [
        # one sequence being generated alone: latency is all there is
        ("norm_rope_single", _case("norm_rope", "1b", "bf16", 1, 1, 2000)),
        # the paper's fp32 prompts (its small-GPU batch)
        ("norm_rope_f32", _case("norm_rope", "paper", "f32", 4, 1024)),
        # a packed batch of prompts, straight out of one wide projection
        ("norm_rope_prompts", _case("norm_rope", "1b", "bf16", 8, 4096, shortest=500, fused=True, mix=1)),
        # a serving batch's decode step: one row per sequence into pages
        ("append_step", _case("append", "1b", "bf16", 64, 1, 4000, shortest=100, page=64, mix=2)),
        # the rows of a batch of prompts, in 16 bits and, as the paper times its layer first, in 32
        ("append_prompts", _case("append", "1b", "bf16", 8, 4096, shortest=500, mix=3)),
        ("append_prompts_f32", _case("append", "paper", "f32", 32, 2048, page=16, mix=4)),
        # cached conversations are read back before new tokens are run behind them
        ("read_prefix", _case("read", "1b", "bf16", 8, 8192, shortest=1200, page=64, mix=5)),
        # decode of one sequence, of the paper's server batch in both precisions, of a 1B-class serving batch, and of
        # long ragged contexts in pages
        ("attend_single", _case("attend", "paper", "bf16", 1, 1, 1000)),
        ("attend_paper", _case("attend", "paper", "bf16", 64, 1, 2048)),
        ("attend_paper_f32", _case("attend", "paper", "f32", 64, 1, 2048)),
        ("attend_batch", _case("attend", "1b", "bf16", 64, 1, 8192)),
        ("attend_long_paged", _case("attend", "wide", "bf16", 8, 1, 32768, shortest=8000, page=64, mix=6)),
    ]
    return [dict(c, name=name) for name, c in cases]


def _log(rng: random.Random, lo: int, hi: int) -> int:
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random) -> Dict:
    """Another case of the same ranges; sizes are capped so that none costs more than the largest listed one."""
    kind = rng.choice(["norm_rope", "append", "read", "attend", "attend"])
    layer, dtype = rng.choice(["paper", "paper768", "1b", "wide"]), rng.choice(["bf16", "bf16", "f32"])
    page, mix = rng.choice([0, 0, 16, 64]), rng.randrange(1 << 16)
    narrow = layer.startswith("paper")

    def low(n: int) -> int:
        return max(1, n // rng.choice([2, 4, 8])) if rng.random() < 0.6 else 0

    if kind == "attend":
        n = _log(rng, 1, 32768)
        most = (1 << 20 if narrow else 1 << 19 if layer == "1b" else 1 << 18) // (2 if dtype == "f32" else 1)
        return _case(kind, layer, dtype, _log(rng, 1, max(1, min(256, most // n))), 1, n, shortest=low(n), page=page, mix=mix)
    cached = _log(rng, 1, 8192)
    if rng.random() < 0.4:   # decode steps and short pieces
        n, batch = rng.choice([1, 1, 1, rng.randint(2, 9)]), _log(rng, 1, 300)
        cached = min(cached, 262144 // batch)
    else:
        n = _log(rng, 16, 8192)
        batch = _log(rng, 1, max(1, min(64, (32768 if narrow else 16384) // n)))
    return _case(kind, layer, dtype, batch, n, 0 if kind == "read" else cached, shortest=low(n), page=page,
                 fused=rng.random() < 0.5, mix=mix)


# ------------------------------------------------------------------------------------------ sizes
def _lengths(case: Dict):
    """(new rows, rows cached before) of every sequence; the first sequence has the longest of both."""
    b, longest, cached, low = case["batch"], case["new"], case["cached"], case["shortest"]
    rng = random.Random(case["mix"])
    if case["kind"] == "attend":
        return [1] * b, [cached] + [rng.randint(min(low, cached), cached) if low else cached for _ in range(b - 1)]
    spread = [longest] + [rng.randint(min(low, longest), longest) if low else longest for _ in range(b - 1)]
    return spread, [cached] + [rng.randint(0, cached) if low else cached for _ in range(b - 1)]


def _widths(case: Dict):
    L = LAYERS[case["layer"]]
    return L["n_qgroups"] * L["head_dim"], L["n_kgroups"] * L["head_dim"], L["n_cgroups"] * L["latent_dim"]


def _capacity(case: Dict) -> int:
    """Rows of a cache slot: the longest sequence and some room, in whole pages of 64."""
    new, cached = _lengths(case)
    return (max(n + p for n, p in zip(new, cached)) + 64 + 63) // 64 * 64


def work(case: Dict) -> Dict[str, float]:
    L = LAYERS[case["layer"]]
    es = 2 if case["dtype"] == "bf16" else 4
    new, cached = _lengths(case)
    qw, kw, cw = _widths(case)
    dh, dl, nq = L["head_dim"], L["latent_dim"], L["n_qgroups"]
    stored = (kw + cw) * (1 + 1 / BLOCK)
    tokens = sum(new)
    if case["kind"] == "norm_rope":
        return {"bytes": float(tokens * (2 * (qw + kw) * es + 4) + 2 * dh * es), "flops": 10.0 * tokens * (qw + kw)}
    if case["kind"] in ("append", "read"):
        return {"bytes": float(tokens * ((kw + cw) * es + stored)), "flops": 3.0 * tokens * (kw + cw)}
    rows = sum(cached)
    return {"bytes": float(rows * stored + case["batch"] * (qw + nq * dl) * es), "flops": 2.0 * nq * (dh + dl) * rows}


# ------------------------------------------------------------------------------------------ inputs
def _quantise(x: torch.Tensor):
    """[rows, width] in 32 bits -> (e4m3 codes, scale bytes [rows, width / 32])."""
    v = x.view(x.shape[0], -1, BLOCK)
    amax = torch.where(torch.isfinite(v), v.abs(), 0.0).amax(dim=-1)
    mant, expo = torch.frexp(amax)            # amax = mant * 2^expo, mant in [1/2, 1)
    e = torch.where(amax > 0, expo - 9 + (mant > 0.875), -117).clamp(-117, 119)
    y = torch.where(torch.isfinite(v), torch.ldexp(v, -e[..., None]).clamp(-448.0, 448.0), math.nan)
    return y.to(torch.float8_e4m3fn).view(x.shape), (e + 127).to(torch.uint8)


def _values(codes: torch.Tensor, scale: torch.Tensor) -> torch.Tensor:
    """What quantised rows [..., width] stand for, in 32 bits."""
    v = codes.float().unflatten(-1, (-1, BLOCK))
    return torch.ldexp(v, scale.int()[..., None] - 127).flatten(-2)


def _draw_inputs(case: Dict, seed: int) -> Dict:
    """Rows N(0,1) with channels of different size (as keys have them), gains near 1, pages in random order; rows of a
    cache behind a sequence's end are zero."""
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * (seed + 1) + case["mix"])
    L, kind = LAYERS[case["layer"]], case["kind"]
    qw, kw, cw = _widths(case)
    new, cached = _lengths(case)
    b, cap, page, total = case["batch"], _capacity(case), case["page"], sum(new)

    def normal(*shape):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=g)

    s = dict(kind=kind, dtype=dt, batch=b, total=total, longest=max(new), page=page, cap=cap,
             nq=L["n_qgroups"], nk=L["n_kgroups"], nc=L["n_cgroups"], dh=L["head_dim"], dl=L["latent_dim"])
    ends = torch.tensor([0] + new, dtype=torch.int64, device="cuda").cumsum(0)
    s["cu"] = ends.to(torch.int32)
    s["start"] = torch.tensor(cached, dtype=torch.int32, device="cuda")
    s["seq"] = torch.repeat_interleave(torch.arange(b, device="cuda"), torch.tensor(new, device="cuda"))
    s["pos"] = torch.arange(total, device="cuda") - ends[s["seq"]] + s["start"][s["seq"]]
    if kind == "norm_rope":
        s["positions"] = s["pos"].to(torch.int32)
        widths = [qw, kw, cw, L["n_heads"] * L["head_dim"]] if case["fused"] else [qw, kw]
        rows = (normal(total, sum(widths)) * (0.4 * normal(1, sum(widths))).exp()).to(dt)
        s["rows"], s["q"], s["k"] = rows, rows[:, :qw], rows[:, qw:qw + kw]
        if not case["fused"]:
            s["q"], s["k"] = s["q"].contiguous(), s["k"].contiguous()
        s["q_gain"], s["k_gain"] = ((1 + 0.2 * normal(L["head_dim"])).to(dt) for _ in range(2))
        return s
    if kind == "append":
        cols = kw + cw + (qw if case["fused"] else 0)
        rows = (normal(total, cols) * (0.4 * normal(1, cols)).exp()).to(dt)
        s["rows"], s["k_new"], s["c_new"] = rows, rows[:, cols - kw - cw:cols - cw], rows[:, cols - cw:]
        if not case["fused"]:
            s["k_new"], s["c_new"] = s["k_new"].contiguous(), s["c_new"].contiguous()
    if page:
        perm = torch.randperm(b * (cap // page), generator=torch.Generator().manual_seed(seed + 17))
        s["table"] = perm.to(torch.int32).view(b, -1).cuda()
    else:
        s["table"] = None
    shape = (b * (cap // page), page) if page else (b, cap)
    for name, width in (("k", kw), ("c", cw)):
        if kind == "append":
            codes = torch.zeros((b * cap, width), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
            scale = torch.zeros((b * cap, width // BLOCK), dtype=torch.uint8, device="cuda")
        else:
            codes, scale = _quantise(normal(b * cap, width) * (0.4 * normal(1, width)).exp())
        s[name], s[name + "_scale"] = codes.view(*shape, width), scale.view(*shape, width // BLOCK)
    lens = s["start"] if kind != "read" else torch.tensor(new, dtype=torch.int32, device="cuda")
    s["lens"] = lens
    if kind != "append":
        row = torch.arange(cap, device="cuda")[None, :]
        at = _rows_of(s, torch.arange(b, device="cuda")[:, None].expand(b, cap), row.expand(b, cap))[row >= lens[:, None]]
        for name in ("k", "c"):
            s[name].view(torch.uint8).view(b * cap, -1)[at] = 0
    if kind == "attend":
        s["q"] = normal(b, qw).to(dt)
    return s


def _rows_of(s: Dict, seq: torch.Tensor, pos: torch.Tensor) -> torch.Tensor:
    """Pool row of row `pos` of sequence `seq`."""
    if s["table"] is None:
        return seq * s["cap"] + pos
    return s["table"].long()[seq, pos // s["page"]] * s["page"] + pos % s["page"]


def prepare(case: Dict, seed: int) -> Dict:
    L = LAYERS[case["layer"]]
    s = _draw_inputs(case, seed)
    kind, dt, total, b = s["kind"], s["dtype"], s["total"], s["batch"]
    if kind != "norm_rope":
        s["seq_lens"], s["status"] = s["lens"].clone(), torch.zeros_like(s["lens"])

    def empty(*shape):
        return torch.empty(shape, dtype=dt, device="cuda")

    if kind == "norm_rope":
        s["q_out"], s["k_out"] = empty(total, s["nq"] * s["dh"]), empty(total, s["nk"] * s["dh"])
    elif kind == "read":
        s["k_out"], s["c_out"] = empty(total, s["nk"] * s["dh"]), empty(total, s["nc"] * s["dl"])
    elif kind == "attend":
        s["l_out"] = empty(b, s["nq"] * s["dl"])
    if own:
        from paper_2506_17286_amd import binding as B
        s["B"], s["cfg"] = B, B.make_config(dtype=case["dtype"], rope=True, rope_base=ROPE_BASE, **L)
        if kind != "norm_rope":
            parts = (s["k"], s["c"], s["k_scale"], s["c_scale"], s["seq_lens"], s["status"])
            s["cache"] = B.make_paged_mx_cache(*parts, s["table"]) if s["page"] else B.make_mx_cache(*parts)
        if kind == "attend":
            s["ws"] = B.alloc_workspace(B.gta_workspace_bytes(s["cfg"], B.GTA_MODE_MX_DECODE, b, 0, s["cap"]))
    return s


# ------------------------------------------------------------------------------------------ the operators
def _plain_norm_rope(s: Dict, x: torch.Tensor, gain: torch.Tensor, heads: int) -> torch.Tensor:
    v = x.float().view(s["total"], heads, s["dh"])
    v = v * torch.rsqrt(v.square().mean(dim=-1, keepdim=True) + EPS) * gain.float()
    half = s["dh"] // 2
    theta = ROPE_BASE ** (-torch.arange(half, dtype=torch.float64, device=x.device) / half)
    angle = (s["positions"].double()[:, None] * theta)[:, None, :]
    cos, sin = angle.cos().float(), angle.sin().float()
    lo, hi = v[..., :half], v[..., half:]
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1).view(s["total"], -1).to(s["dtype"])


def _plain_attend(s: Dict) -> torch.Tensor:
    b, nq, nk, nc, dh, dl, cap = (s[n] for n in ("batch", "nq", "nk", "nc", "dh", "dl", "cap"))

    def cached(name):
        codes, scale = s[name].view(torch.uint8), s[name + "_scale"]
        if s["table"] is not None:
            at = s["table"].long()
            codes, scale = codes[at], scale[at]
        return _values(codes.view(torch.float8_e4m3fn), scale).reshape(b, cap, -1)

    k = cached("k").view(b, cap, nk, dh).permute(0, 2, 3, 1).contiguous()          # [b, nk, dh, cap]
    score = (s["q"].float().view(b, nk, nq // nk, dh) @ k).view(b, nq, cap) / math.sqrt(dh)
    score = score.masked_fill(torch.arange(cap, device=k.device) >= s["seq_lens"][:, None, None], -math.inf)
    p = (score - score.amax(dim=-1, keepdim=True)).exp()
    p = p / p.sum(dim=-1, keepdim=True)
    c = cached("c").view(b, cap, nc, dl).transpose(1, 2).contiguous()
    return (p.view(b, nc, nq // nc, cap) @ c).view(b, nq * dl).to(s["dtype"])


def run(s: Dict) -> Dict:
    kind = s["kind"]
    if kind == "norm_rope":
        if own:
            s["B"].gta_qk_norm_rope(s["cfg"], s["q"], s["q"].stride(0), s["k"], s["k"].stride(0), s["q_gain"], s["k_gain"], EPS,
                                    s["positions"], s["total"], s["q_out"], s["k_out"])
            return {"q": s["q_out"], "k": s["k_out"]}
        return {"q": _plain_norm_rope(s, s["q"], s["q_gain"], s["nq"]), "k": _plain_norm_rope(s, s["k"], s["k_gain"], s["nk"])}
    if kind == "append":
        # every pass starts from the same cached lengths: one small kernel where a serving loop sets its lengths
        torch.add(s["start"], 0, out=s["seq_lens"])
        if own:
            s["B"].gta_mx_cache_append(s["cfg"], s["cache"], None, s["k_new"], s["k_new"].stride(0), s["c_new"], s["c_new"].stride(0),
                                       s["cu"], s["batch"], s["longest"])
        else:
            at = _rows_of(s, s["seq"], s["pos"])
            for name, rows in (("k", s["k_new"]), ("c", s["c_new"])):
                codes, scale = _quantise(rows.float().contiguous())
                s[name].view(torch.uint8).view(-1, codes.shape[1])[at] = codes.view(torch.uint8)
                s[name + "_scale"].view(-1, scale.shape[1])[at] = scale
            s["seq_lens"] += s["cu"][1:] - s["cu"][:-1]
        return {n: s[n] for n in ("k", "c", "k_scale", "c_scale", "seq_lens", "status")}
    if kind == "read":
        if own:
            s["B"].gta_mx_cache_read(s["cfg"], s["cache"], None, None, s["cu"], s["batch"], s["longest"], s["k_out"], s["c_out"])
            return {"k": s["k_out"], "c": s["c_out"]}
        at, out = _rows_of(s, s["seq"], s["pos"]), {}
        for name in ("k", "c"):
            codes = s[name].view(torch.uint8).view(-1, s[name].shape[-1])[at].view(torch.float8_e4m3fn)
            out[name] = _values(codes, s[name + "_scale"].view(-1, s[name + "_scale"].shape[-1])[at]).to(s["dtype"])
        return out
    if own:
        s["B"].gta_mx_decode_attention(s["cfg"], s["q"], s["cache"], None, s["batch"], 0, s["l_out"], s["ws"])
        return {"l": s["l_out"]}
    return {"l": _plain_attend(s)}


# ------------------------------------------------------------------------------------------ 64-bit answer
def _exact_quantise(x: torch.Tensor):
    """Codes (as the numbers they are) and scale bytes, by arithmetic on float64."""
    v = x.double().reshape(x.shape[0], -1, BLOCK)
    top = v.abs().amax(dim=-1)
    e = torch.full_like(top, -117.0)
    some = top > 0
    e[some] = torch.ceil(torch.log2(top[some] / 448.0))
    e = torch.where(top > 448.0 * torch.exp2(e), e + 1, e)                  # the logarithm's own rounding
    e = torch.where(some & (top <= 448.0 * torch.exp2(e - 1)), e - 1, e).clamp(-117, 119)
    y = (v / torch.exp2(e)[..., None]).clamp(-448.0, 448.0)
    expo = torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6)))
    step = torch.exp2(expo - 3)                                             # 3 bits behind the leading one; 2^-9 at the bottom
    return (torch.round(y / step) * step).reshape(x.shape), (e + 127).to(torch.uint8)


def exact(case: Dict, seed: int) -> Dict:
    s = _draw_inputs(case, seed)
    kind, b, dh, dl, nq, nk, nc = (s[n] for n in ("kind", "batch", "dh", "dl", "nq", "nk", "nc"))
    if kind == "norm_rope":
        out = {}
        j = torch.arange(dh // 2, dtype=torch.float64, device="cuda")
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * ROPE_BASE ** (-2 * j / dh))
        for name, heads in (("q", nq), ("k", nk)):
            x = s[name].double().reshape(-1, heads, dh)
            x = x / (x.square().sum(-1, keepdim=True) / dh + EPS).sqrt() * s[name + "_gain"].double()
            z = torch.complex(x[..., :dh // 2].contiguous(), x[..., dh // 2:].contiguous()) * turn[:, None, :]
            out[name] = torch.cat([z.real, z.imag], dim=-1).reshape(s["total"], heads * dh)
        return out
    cap = s["cap"]

    def stored(name, i, n):
        """rows 0 .. n-1 of sequence i, in float64"""
        rows = torch.arange(n, device="cuda")
        rows = s["table"][i].long()[rows // s["page"]] * s["page"] + rows % s["page"] if s["page"] else rows + i * cap
        codes = s[name].view(torch.uint8).view(b * cap, -1)[rows].view(torch.float8_e4m3fn).double()
        return codes * torch.exp2(s[name + "_scale"].view(b * cap, -1)[rows].double() - 127).repeat_interleave(BLOCK, dim=1)

    if kind == "append":
        out = {"seq_lens": s["start"] + (s["cu"][1:] - s["cu"][:-1]), "status": torch.zeros_like(s["start"])}
        at = _rows_of(s, s["seq"], s["pos"])
        for name, rows in (("k", s["k_new"]), ("c", s["c_new"])):
            codes = s[name].double().view(b * cap, -1)
            codes[at], s[name + "_scale"].view(b * cap, -1)[at] = _exact_quantise(rows)
            out[name], out[name + "_scale"] = codes.view(s[name].shape), s[name + "_scale"]
        return out
    lens = s["lens"].tolist()
    if kind == "read":
        return {name: torch.cat([stored(name, i, n) for i, n in enumerate(lens)]) for name in ("k", "c")}
    out = torch.zeros((b, nq, dl), dtype=torch.float64, device="cuda")
    for i, n in enumerate(lens):
        k, c = stored("k", i, n).view(n, nk, dh), stored("c", i, n).view(n, nc, dl)
        for g in range(nq):
            a = k[:, g * nk // nq].contiguous() @ s["q"][i, g * dh:(g + 1) * dh].double() / math.sqrt(dh)
            out[i, g] = torch.softmax(a, dim=0) @ c[:, g * nc // nq].contiguous()
    return {"l": out.view(b, nq * dl)}
