"""Operators around long and structured contexts, as measurable cases.

One case is one pass through one operator on tensors that already live on the GPU:

  rope    rotary positions of projected queries and keys: pairs (j, j + r/2) or (2j, 2j + 1) of the first r elements of a
          head, frequencies as trained or scaled for longer contexts, forwards or transposed (the gradient's direction)
  masked  attention of a packed batch whose scores may be capped by a tanh and get a bias that falls with the distance, every
          token seeing an interval of its sequence: documents packed together, a prefix seen from everywhere, a window
  prefix  one new token per sequence attends over a prefix that the whole batch shares and over its own cached rows

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
TRAINED, SLOW, FAST = 4096, 1.0, 4.0     # bands: length of the training, turns over it below / above which a pair is scaled / kept


def _case(kind: str, layer: str, dtype: str, batch: int, longest: int, shortest: int = 0, mix: int = 0, **more) -> Dict:
    """longest: tokens of the longest sequence (rope, masked) or rows of its own in the cache (prefix); shortest > 0:
    lengths spread over [shortest, longest] by the generator `mix`.  rope: layout, part (the head's elements over those that
    turn), scaling, factor, offset (position of each sequence's first token), fused (rows are columns of one wide
    projection's output), back (transposed).  masked, prefix: cap and bias of the scores; masked: mask and its size;
    prefix: rows of the prefix, page (rows of a page, 0 for contiguous slots)."""
    base = dict(kind=kind, layer=layer, dtype=dtype, batch=batch, longest=longest, shortest=shortest, mix=mix)
    if kind == "rope":
        base.update(layout="half", part=1, scaling="plain", factor=1.0, offset=0, fused=False, back=False)
    else:
        base.update(cap=0.0, bias=False)
        base.update(dict(mask="causal", size=0, fused=False) if kind == "masked" else dict(prefix=0, page=0))
    base.update(more)
    return base


def listed() -> List[Dict]:
    cases = [
        # one sequence being generated alone, far behind the trained length: latency is all there is
        ("rope_single", _case("rope", "1b", "bf16", 1, 1, scaling="bands", factor=8.0, offset=20000)),
        # a packed batch of prompts straight out of one wide projection; half of each head turns, neighbours in pairs
        ("rope_prompts", _case("rope", "1b", "bf16", 8, 4096, 500, 1, layout="interleaved", part=2, scaling="linear", factor=4.0,
                               fused=True)),
        # the gradient's direction in the paper's first precision (its small-GPU batch)
        ("rope_back_f32", _case("rope", "paper", "f32", 4, 1024, scaling="base", factor=4.0, back=True)),
        # a chat turn of a few dozen tokens with capped scores: latency
        ("masked_short", _case("masked", "paper", "bf16", 1, 60, cap=30.0)),
        # documents of 100 to 2000 tokens packed into rows of 4096, as they are trained and scored
        ("masked_documents", _case("masked", "1b", "bf16", 4, 4096, 0, 2, mask="documents", size=2000)),
        # instructions of up to a half of the prompt seen from everywhere, ragged prompts, capped scores
        ("masked_prefix_cap", _case("masked", "paper", "bf16", 32, 2048, 300, 3, mask="prefix", size=1000, cap=30.0)),
        # distance instead of positions, in 32 bits
        ("masked_bias_f32", _case("masked", "paper", "f32", 4, 1024, bias=True)),
        # two long contexts under a window, distances and capped scores together
        ("masked_window", _case("masked", "wide", "bf16", 2, 8192, 7000, 4, mask="window", size=4096, cap=50.0, bias=True)),
        # two continuations of one short prompt
        ("prefix_single", _case("prefix", "paper", "bf16", 2, 20, prefix=1000)),
        # a serving batch behind one long system prompt, capped scores, conversations of different length
        ("prefix_batch", _case("prefix", "1b", "bf16", 64, 1500, 20, 5, prefix=8192, cap=30.0)),
        # the paper's server batch in 32 bits with distances
        ("prefix_f32", _case("prefix", "paper", "f32", 64, 256, prefix=2048, bias=True)),
        # many readers of one very long document, everything in pages
        ("prefix_long_paged", _case("prefix", "wide", "bf16", 32, 4000, 100, 6, prefix=32768, page=64)),
    ]
    return [dict(c, name=name) for name, c in cases]


def _log(rng: random.Random, lo: int, hi: int) -> int:
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random) -> Dict:
    """Another case of the same ranges; sizes are capped so that none costs more than the largest listed one."""
    kind = rng.choice(["rope", "masked", "masked", "prefix", "prefix"])
    layer, dtype = rng.choice(["paper", "paper768", "1b", "wide"]), rng.choice(["bf16", "bf16", "f32"])
    mix, narrow = rng.randrange(1 << 16), layer.startswith("paper")

    def low(n: int) -> int:
        return max(1, n // rng.choice([2, 4, 8])) if rng.random() < 0.6 else 0

    if kind == "rope":
        n = 1 if rng.random() < 0.3 else _log(rng, 2, 8192)
        batch = _log(rng, 1, max(1, min(256, (32768 if narrow else 16384) // n)))
        scaling = rng.choice(["plain", "linear", "base", "bands"])
        return _case(kind, layer, dtype, batch, n, low(n), mix, layout=rng.choice(["half", "interleaved"]), part=rng.choice([1, 1, 2, 4]),
                     scaling=scaling, factor=1.0 if scaling == "plain" else rng.choice([2.0, 4.0, 8.0, 32.0]),
                     offset=_log(rng, 1, 100000) - 1, fused=rng.random() < 0.5, back=rng.random() < 0.4)
    cap, bias = rng.choice([0.0, 0.0, 20.0, 50.0]), rng.random() < 0.4
    if kind == "masked":
        n = _log(rng, 1, (8192 if narrow or layer == "1b" else 4096) // (2 if dtype == "f32" else 1))
        most = (1 << 16 if narrow else 1 << 14 if layer == "1b" else 1 << 13) // (4 if dtype == "f32" else 1)
        batch = _log(rng, 1, max(1, min(128, most // n)))
        mask = rng.choice(["causal", "documents", "prefix", "window", "whole"])
        return _case(kind, layer, dtype, batch, n, low(n), mix, cap=cap, bias=bias, mask=mask, size=_log(rng, 1, n),
                     fused=rng.random() < 0.5)
    n = _log(rng, 1, 4096)
    rows = 1 << (19 if narrow else 18 if layer == "1b" else 17) - (dtype == "f32")
    batch = _log(rng, 1, max(1, min(256, rows // n)))
    top = 32768 if narrow or batch <= 64 else 8192
    return _case(kind, layer, dtype, batch, n, low(n), mix, cap=cap, bias=bias, prefix=_log(rng, 1, top // (2 if dtype == "f32" else 1)),
                 page=rng.choice([0, 0, 16, 64]))


# ------------------------------------------------------------------------------------------ sizes
def _lengths(case: Dict) -> List[int]:
    """The first sequence is the longest."""
    rng, n, low = random.Random(case["mix"]), case["longest"], case["shortest"]
    return [n] + [rng.randint(min(low, n), n) if low else n for _ in range(case["batch"] - 1)]


def _widths(case: Dict):
    L = LAYERS[case["layer"]]
    return L["n_qgroups"] * L["head_dim"], L["n_kgroups"] * L["head_dim"], L["n_cgroups"] * L["latent_dim"]


def _capacity(case: Dict) -> int:
    return (case["longest"] + 64 + 63) // 64 * 64


def _intervals(case: Dict):
    """First and last token that each token sees, sequence by sequence."""
    rng, mask, size = random.Random(case["mix"] + 77), case["mask"], case["size"]
    first, last = [], []
    for n in _lengths(case):
        lo, hi = [0] * n, list(range(n))
        if mask == "documents":
            at = 0
            while at < n:
                end = min(n, at + rng.randint(max(1, size // 20), size))
                lo[at:end] = [at] * (end - at)
                at = end
        elif mask == "prefix":
            seen = rng.randint(0, min(size, n))
            hi = [max(i, seen - 1) for i in range(n)]
        elif mask == "window":
            lo = [max(0, i - size + 1) for i in range(n)]
        elif mask == "whole":
            hi = [n - 1] * n
        first += lo
        last += hi
    return first, last


def work(case: Dict) -> Dict[str, float]:
    L = LAYERS[case["layer"]]
    es = 2 if case["dtype"] == "bf16" else 4
    qw, kw, cw = _widths(case)
    dh, dl, nq, b = L["head_dim"], L["latent_dim"], L["n_qgroups"], case["batch"]
    lens = _lengths(case)
    tokens = sum(lens)
    if case["kind"] == "rope":
        return {"bytes": float(tokens * (2 * (qw + kw) * es + 4)), "flops": 3.0 * tokens * (qw + kw)}
    if case["kind"] == "masked":
        first, last = _intervals(case)
        seen = sum(hi - lo + 1 for lo, hi in zip(first, last))
        return {"bytes": float(tokens * ((qw + kw + cw + nq * dl) * es + 8)), "flops": 2.0 * nq * (dh + dl) * seen}
    rows = case["prefix"] + tokens
    return {"bytes": float(rows * (kw + cw) * es + b * (qw + nq * dl) * es), "flops": 2.0 * nq * (dh + dl) * (b * case["prefix"] + tokens)}


# ------------------------------------------------------------------------------------------ inputs
def _draw_inputs(case: Dict, seed: int) -> Dict:
    """Rows N(0,1) with channels of different size (as keys have them); queries that give scores of a few units; pages in
    random order; what lies behind a sequence's end in a cache is zero."""
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * (seed + 1) + case["mix"])
    L, kind = LAYERS[case["layer"]], case["kind"]
    qw, kw, cw = _widths(case)
    lens, b = _lengths(case), case["batch"]
    total = sum(lens)

    def normal(*shape):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=g)

    def rows(n, width):
        return normal(n, width) * (0.3 * normal(1, width)).exp()

    s = dict(kind=kind, dtype=dt, batch=b, total=total, longest=case["longest"], nq=L["n_qgroups"], nk=L["n_kgroups"],
             nc=L["n_cgroups"], dh=L["head_dim"], dl=L["latent_dim"], case=case)
    ends = torch.tensor([0] + lens, dtype=torch.int64, device="cuda").cumsum(0)
    s["cu"], s["lens"], s["lengths"] = ends.to(torch.int32), torch.tensor(lens, dtype=torch.int32, device="cuda"), lens
    if kind != "prefix":
        seq = torch.repeat_interleave(torch.arange(b, device="cuda"), torch.tensor(lens, device="cuda"))
        s["index"] = torch.arange(total, device="cuda") - ends[seq]
    if kind == "rope":
        s["positions"] = (s["index"] + case["offset"]).to(torch.int32)
        wide = rows(total, qw + kw + (cw if case["fused"] else 0)).to(dt)
        s["rows"], s["q"], s["k"] = wide, wide[:, :qw], wide[:, qw:qw + kw]
        if not case["fused"]:
            s["q"], s["k"] = s["q"].contiguous(), s["k"].contiguous()
        return s
    s["cap"] = case["cap"]
    s["slopes"] = torch.exp2(-8.0 * torch.arange(1, s["nq"] + 1, device="cuda") / s["nq"]) if case["bias"] else None
    if kind == "masked":
        wide = rows(total, qw + kw + cw)
        wide[:, :qw] *= 2.0
        wide = wide.to(dt)
        s["rows"], s["q"], s["k"], s["c"] = wide, wide[:, :qw], wide[:, qw:qw + kw], wide[:, qw + kw:]
        if not case["fused"]:
            s["q"], s["k"], s["c"] = s["q"].contiguous(), s["k"].contiguous(), s["c"].contiguous()
        first, last = _intervals(case)
        s["first"], s["last"] = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (first, last))
        return s
    page, cap = case["page"], _capacity(case)
    s["page"], s["room"] = page, cap
    s["q"] = (rows(b, qw) * 2.0).to(dt)
    s["prefix_rows"] = case["prefix"]
    s["prefix_room"] = (case["prefix"] + 63) // 64 * 64
    s["prefix_len"] = torch.tensor([case["prefix"]], dtype=torch.int32, device="cuda")
    perm = torch.Generator().manual_seed(seed + 17)
    for name, slots, room in (("prefix_", 1, s["prefix_room"]), ("", b, cap)):
        s[name + "table"] = torch.randperm(slots * (room // page), generator=perm).to(torch.int32).view(slots, -1).cuda() if page else None
        shape = (slots * (room // page), page) if page else (slots, room)
        n = s["prefix_len"] if name else s["lens"]
        row = torch.arange(room, device="cuda")[None, :].expand(slots, room)
        at = _rows_of(s, name, torch.arange(slots, device="cuda")[:, None].expand(slots, room), row)[row >= n[:, None]]
        for part, width in (("k", kw), ("c", cw)):
            pool = rows(slots * room, width).to(dt)
            pool[at] = 0
            s[name + part] = pool.view(*shape, width)
    return s


def _rows_of(s: Dict, name: str, slot: torch.Tensor, pos: torch.Tensor) -> torch.Tensor:
    """Pool row of row `pos` of a slot of the prefix's (name "prefix_") or the sequences' (name "") cache."""
    table, page = s[name + "table"], s["page"]
    if table is None:
        return slot * s[name + "room"] + pos
    return table.long()[slot, pos // page] * page + pos % page


def prepare(case: Dict, seed: int) -> Dict:
    L = LAYERS[case["layer"]]
    s = _draw_inputs(case, seed)
    kind, dt = s["kind"], s["dtype"]

    def empty(*shape):
        return torch.empty(shape, dtype=dt, device="cuda")

    if kind == "rope":
        s["q_out"], s["k_out"] = empty(s["total"], s["nq"] * s["dh"]), empty(s["total"], s["nk"] * s["dh"])
    else:
        s["l_out"] = empty(s["total"] if kind == "masked" else s["batch"], s["nq"] * s["dl"])
    if own:
        from paper_2506_17286_amd import binding as B
        s["B"], cfg = B, B.make_config(dtype=case["dtype"], **L)
        s["cfg"] = cfg
        if kind == "rope":
            s["rotation"] = B.make_rotation(cfg, layout=case["layout"], rotary_dim=s["dh"] // case["part"], base=ROPE_BASE,
                                            scaling=case["scaling"], factor=case["factor"], trained_len=TRAINED, slow_turns=SLOW,
                                            fast_turns=FAST)
        elif kind == "masked":
            causal = case["mask"] == "causal"
            s["rules"] = B.make_score_rules(cap=s["cap"], slopes=s["slopes"], first=None if causal else s["first"],
                                            last=None if causal else s["last"])
            s["ws"] = B.alloc_workspace(B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFILL_MASKED, s["batch"], s["total"], s["longest"]))
        else:
            s["rules"] = B.make_score_rules(cap=s["cap"], slopes=s["slopes"])
            s["status"], s["prefix_status"] = torch.zeros_like(s["lens"]), torch.zeros_like(s["prefix_len"])
            for name, lens in (("prefix_", s["prefix_len"]), ("", s["lens"])):
                parts = (s[name + "k"], s[name + "c"], lens, s[name + "status"])
                s[name + "cache"] = B.make_paged_cache(*parts, s[name + "table"]) if s["page"] else B.make_cache(*parts)
            s["ws"] = B.alloc_workspace(B.gta_workspace_bytes(cfg, B.GTA_MODE_PREFIX_DECODE, s["batch"], s["prefix_room"], s["room"]))
    return s


# ------------------------------------------------------------------------------------------ the operators
def _frequencies(case: Dict, r: int, device) -> torch.Tensor:
    """Radians that one position turns each pair by, in 64 bits."""
    j = torch.arange(r // 2, dtype=torch.float64, device=device)
    s = case["factor"]
    base = ROPE_BASE * s ** (r / (r - 2)) if case["scaling"] == "base" else ROPE_BASE
    f = base ** (-2.0 * j / r)
    if case["scaling"] == "linear":
        return f / s
    if case["scaling"] == "bands":
        keep = ((TRAINED * f / (2 * math.pi) - SLOW) / (FAST - SLOW)).clamp(0.0, 1.0)
        return (1 - keep) * f / s + keep * f
    return f


def _plain_rope(s: Dict, x: torch.Tensor, heads: int) -> torch.Tensor:
    case, dh = s["case"], s["dh"]
    r = dh // case["part"]
    angle = (s["positions"].double()[:, None] * _frequencies(case, r, x.device))[:, None, :]
    cos, sin = angle.cos().float(), angle.sin().float()
    if case["back"]:
        sin = -sin
    v = x.float().reshape(s["total"], heads, dh)
    if case["layout"] == "half":
        lo, hi = v[..., :r // 2], v[..., r // 2:r]
        turned = torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1)
    else:
        lo, hi = v[..., 0:r:2], v[..., 1:r:2]
        turned = torch.stack([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1).flatten(-2)
    return torch.cat([turned, v[..., r:]], dim=-1).view(s["total"], -1).to(s["dtype"])


def _plain_softmax(s: Dict, score: torch.Tensor, distance: torch.Tensor, seen: torch.Tensor) -> torch.Tensor:
    """Scaled scores [.., maps, keys] -> weights; distance and seen broadcast over the maps."""
    if s["cap"]:
        score = s["cap"] * torch.tanh(score / s["cap"])
    if s["slopes"] is not None:
        score = score - s["slopes"][:, None] * distance.float()
    score = score.masked_fill(~seen, -math.inf)
    p = (score - score.amax(dim=-1, keepdim=True)).exp()
    return p / p.sum(dim=-1, keepdim=True)


def _plain_masked(s: Dict) -> torch.Tensor:
    nq, nk, nc, dh, dl = (s[n] for n in ("nq", "nk", "nc", "dh", "dl"))
    out = torch.empty((s["total"], nq * dl), dtype=s["dtype"], device="cuda")
    at = 0
    for n in s["lengths"]:
        rows = slice(at, at + n)
        q = s["q"][rows].float().view(n, nk, nq // nk, dh).permute(1, 2, 0, 3).reshape(nk, nq // nk * n, dh)
        k = s["k"][rows].float().view(n, nk, dh).permute(1, 2, 0).contiguous()
        score = (q @ k).view(nq, n, n).transpose(0, 1) / math.sqrt(dh)              # [token, map, key]
        i, j = torch.arange(n, device="cuda")[:, None, None], torch.arange(n, device="cuda")[None, None, :]
        seen = (j >= s["first"][rows][:, None, None]) & (j <= s["last"][rows][:, None, None])
        p = _plain_softmax(s, score, (i - j).abs(), seen)
        c = s["c"][rows].float().view(n, nc, dl).transpose(0, 1).contiguous()
        p = p.view(n, nc, nq // nc, n).permute(1, 0, 2, 3).reshape(nc, n * (nq // nc), n)
        out[rows] = (p @ c).view(nc, n, nq // nc, dl).transpose(0, 1).reshape(n, nq * dl).to(s["dtype"])
        at += n
    return out


def _plain_prefix(s: Dict) -> torch.Tensor:
    b, nq, nk, nc, dh, dl, rows = (s[n] for n in ("batch", "nq", "nk", "nc", "dh", "dl", "prefix_rows"))

    def cached(name, part):
        pool = s[name + part]
        return (pool if s[name + "table"] is None else pool[s[name + "table"].long()].flatten(1, 2)).float()

    n, room = s["lens"][:, None, None], s["room"]
    q = s["q"].float().view(b, nk, nq // nk, dh)
    shared = cached("prefix_", "k")[0, :rows].reshape(rows, nk, dh).permute(1, 2, 0).contiguous()          # [nk, dh, rows]
    mine = cached("", "k").view(b, room, nk, dh).permute(0, 2, 3, 1).contiguous()
    score = torch.cat([(q.transpose(0, 1).reshape(nk, -1, dh) @ shared).view(nk, b, nq // nk, rows).transpose(0, 1).reshape(b, nq, rows),
                       (q @ mine).view(b, nq, room)], dim=-1) / math.sqrt(dh)
    j = torch.arange(rows + room, device="cuda")
    p = _plain_softmax(s, score, rows + n - 1 - j, j < rows + n)
    p = p.view(b, nc, nq // nc, rows + room)
    shared = cached("prefix_", "c")[0, :rows].reshape(rows, nc, dl).transpose(0, 1).contiguous()
    mine = cached("", "c").view(b, room, nc, dl).transpose(1, 2).contiguous()
    out = (p[..., :rows].transpose(0, 1).reshape(nc, -1, rows) @ shared).view(nc, b, nq // nc, dl).transpose(0, 1)
    return (out + p[..., rows:].contiguous() @ mine).reshape(b, nq * dl).to(s["dtype"])


def run(s: Dict) -> Dict:
    kind = s["kind"]
    if kind == "rope":
        if own:
            s["B"].gta_qk_rope(s["cfg"], s["rotation"], s["q"], s["q"].stride(0), s["k"], s["k"].stride(0), s["positions"], s["total"],
                               s["case"]["back"], s["q_out"], s["q_out"].stride(0), s["k_out"], s["k_out"].stride(0))
            return {"q": s["q_out"], "k": s["k_out"]}
        return {"q": _plain_rope(s, s["q"], s["nq"]), "k": _plain_rope(s, s["k"], s["nk"])}
    if kind == "masked":
        if own:
            s["B"].gta_prefill_masked_attention(s["cfg"], s["q"], s["q"].stride(0), s["k"], s["k"].stride(0), s["c"], s["c"].stride(0),
                                                s["cu"], s["batch"], s["total"], s["longest"], s["rules"], s["l_out"], s["ws"])
            return {"l": s["l_out"]}
        return {"l": _plain_masked(s)}
    if own:
        s["B"].gta_prefix_decode_attention(s["cfg"], s["q"], s["prefix_cache"], 0, s["cache"], None, s["batch"], s["rules"],
                                           s["l_out"], s["ws"])
        return {"l": s["l_out"]}
    return {"l": _plain_prefix(s)}


# ------------------------------------------------------------------------------------------ 64-bit answer
def _exact_rope(s: Dict, x: torch.Tensor, heads: int) -> torch.Tensor:
    """Every pair as a complex number times e^(i angle), the frequencies one by one from their definition."""
    case, dh = s["case"], s["dh"]
    r, factor = dh // case["part"], case["factor"]
    freq = []
    for j in range(r // 2):
        f = math.exp(-2.0 * j / r * math.log(ROPE_BASE))
        if case["scaling"] == "base":
            f = math.exp(-2.0 * j / r * (math.log(ROPE_BASE) + r / (r - 2) * math.log(factor)))
        elif case["scaling"] == "linear":
            f /= factor
        elif case["scaling"] == "bands":
            turns = TRAINED * f / (2 * math.pi)
            f *= 1.0 if turns >= FAST else 1 / factor if turns <= SLOW else ((turns - SLOW) + (FAST - turns) / factor) / (FAST - SLOW)
        freq.append(-f if case["back"] else f)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       s["positions"].double()[:, None] * torch.tensor(freq, dtype=torch.float64, device="cuda"))[:, None, :]
    y = x.double().reshape(-1, heads, dh).clone()
    at = (slice(0, r // 2), slice(r // 2, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    z = torch.complex(y[..., at[0]].contiguous(), y[..., at[1]].contiguous()) * turn
    y[..., at[0]], y[..., at[1]] = z.real, z.imag
    return y.reshape(x.shape[0], heads * dh)


def exact(case: Dict, seed: int) -> Dict:
    s = _draw_inputs(case, seed)
    kind, b, dh, dl, nq, nk, nc = (s[n] for n in ("kind", "batch", "dh", "dl", "nq", "nk", "nc"))
    if kind == "rope":
        return {"q": _exact_rope(s, s["q"], nq), "k": _exact_rope(s, s["k"], nk)}

    def attend(g, q, k, c, where, positions, lo, hi):
        """Map g: queries [m, dh] at `where` [m] over rows k [n, dh], c [n, dl] at `positions`, seeing lo .. hi."""
        a = q.double() @ k.double().T.contiguous() / math.sqrt(dh)
        if s["cap"]:
            e = torch.exp(-2.0 * a.abs() / s["cap"])
            a = torch.sign(a) * s["cap"] * (1 - e) / (1 + e)
        if s["slopes"] is not None:
            a -= s["slopes"][g].double() * (where[:, None] - positions[None, :]).abs().double()
        a[(positions[None, :] < lo[:, None]) | (positions[None, :] > hi[:, None])] = -math.inf
        return torch.softmax(a, dim=-1) @ c.double()

    if kind == "masked":
        out = torch.empty((s["total"], nq * dl), dtype=torch.float64, device="cuda")
        at = 0
        for n in s["lengths"]:
            pos = torch.arange(n, device="cuda")
            for g in range(nq):
                kc, cc = g * nk // nq * dh, g * nc // nq * dl
                for i0 in range(0, n, 2048):
                    i1 = min(n, i0 + 2048)
                    rows = slice(at + i0, at + i1)
                    out[rows, g * dl:(g + 1) * dl] = attend(g, s["q"][rows, g * dh:(g + 1) * dh], s["k"][at:at + n, kc:kc + dh],
                                                            s["c"][at:at + n, cc:cc + dl], pos[i0:i1], pos, s["first"][rows], s["last"][rows])
            at += n
        return {"l": out}
    out = torch.empty((b, nq * dl), dtype=torch.float64, device="cuda")
    p = s["prefix_rows"]
    shared = _rows_of(s, "prefix_", torch.zeros(p, dtype=torch.int64, device="cuda"), torch.arange(p, device="cuda"))
    pools = {n: s[n].reshape(-1, s[n].shape[-1]) for n in ("k", "c", "prefix_k", "prefix_c")}
    shared_k, shared_c = pools["prefix_k"][shared], pools["prefix_c"][shared]
    for i, n in enumerate(s["lengths"]):
        mine = _rows_of(s, "", torch.full((n,), i, device="cuda"), torch.arange(n, device="cuda"))
        k, c = torch.cat([shared_k, pools["k"][mine]]), torch.cat([shared_c, pools["c"][mine]])
        pos = torch.arange(p + n, device="cuda")
        for g in range(nq):
            kc, cc = g * nk // nq * dh, g * nc // nq * dl
            out[i, g * dl:(g + 1) * dl] = attend(g, s["q"][i:i + 1, g * dh:(g + 1) * dh], k[:, kc:kc + dh], c[:, cc:cc + dl],
                                                 pos[-1:], pos, pos[:1], pos[-1:])[0]
    return {"l": out}
