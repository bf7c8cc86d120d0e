"""Plain float64 forms of the operators around an 8-bit cache, and caches to run them on."""
from __future__ import annotations

import numpy as np
import torch

from paper_2506_17286_amd import binding as B

BLOCK = 32
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}   # largest rounding error relative to the value
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _e4m3_table() -> np.ndarray:
    """The number each of the 256 codes stands for: sign, 4 exponent bits (bias 7), 3 mantissa bits; no infinities."""
    t = np.empty(256)
    for i in range(256):
        e, m = (i >> 3) & 15, i & 7
        v = np.nan if (e, m) == (15, 7) else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        t[i] = -v if i & 128 else v
    return t


E4M3 = _e4m3_table()


def quantise(x: np.ndarray):
    """float64 [rows, width] -> (what each code stands for, scale bytes), by the definition in include/gta.h."""
    v = x.reshape(x.shape[0], x.shape[1] // BLOCK, BLOCK)
    fin = np.isfinite(v)
    amax = np.where(fin, np.abs(v), 0).max(axis=-1)
    e = np.full(amax.shape, -117)
    for cand in range(119, -118, -1):          # the least exponent that covers the block
        e = np.where(amax <= 448 * 2.0 ** cand, cand, e)
    e = np.where(amax > 448 * 2.0 ** 119, 119, e)
    y = np.clip(np.where(fin, v, 0) * 2.0 ** -e[..., None].astype(float), -448, 448)
    _, ex = np.frexp(y)                        # y = m * 2^ex, m in [1/2, 1)
    step = 2.0 ** (np.maximum(ex - 1, -6) - 3.0)
    return np.where(fin, np.rint(y / step) * step, np.nan).reshape(x.shape), (e + 127).astype(np.uint8)


def values(codes: np.ndarray, scale: np.ndarray) -> np.ndarray:
    """Stored rows (codes as bytes) as float64."""
    return E4M3[codes] * np.repeat(2.0 ** (scale.astype(float) - 127), BLOCK, axis=-1)


def norm_rope(x: np.ndarray, gain, eps: float, pos: np.ndarray, dh: int, base: float, rope: bool):
    """float64 [tokens, heads*dh]; also the magnitude that rounding errors of the rotation go by."""
    v = x.reshape(x.shape[0], -1, dh)
    v = v / np.sqrt((v ** 2).mean(axis=-1, keepdims=True) + eps) * (1.0 if gain is None else gain)
    if not rope:
        return v.reshape(x.shape), np.abs(v).reshape(x.shape)
    half = dh // 2
    ang = (pos[:, None].astype(float) * base ** (-2.0 * np.arange(half) / dh))[:, None, :]
    lo, hi = v[..., :half], v[..., half:]
    y = np.concatenate([lo * np.cos(ang) - hi * np.sin(ang), hi * np.cos(ang) + lo * np.sin(ang)], axis=-1)
    r = np.hypot(lo, hi)
    return y.reshape(x.shape), np.concatenate([r, r], axis=-1).reshape(x.shape)


def shape(nq, nk, nc, dh, dl, nh=None, H=256):
    return dict(d_model=H, n_heads=nh or nq, n_qgroups=nq, n_kgroups=nk, n_cgroups=nc, head_dim=dh, latent_dim=dl)


# the layers of the repository, groupings with several maps per key and several latents, and widths off every grid
SHAPES = {
    "tiny": shape(2, 2, 1, 32, 64), "paper": shape(5, 1, 1, 64, 128), "paper768": shape(3, 1, 1, 64, 128),
    "gta4": shape(10, 1, 2, 64, 128), "1b": shape(4, 4, 1, 128, 512), "q8k4": shape(8, 4, 1, 128, 512),
    "c2": shape(8, 4, 2, 128, 512), "c4": shape(4, 4, 4, 128, 512), "wide": shape(8, 8, 1, 128, 1024),
    "q16": shape(16, 2, 1, 64, 256), "one": shape(1, 1, 1, 128, 128), "mha": shape(20, 20, 20, 64, 64),
    "odd": shape(6, 3, 2, 96, 160), "head256": shape(2, 1, 1, 256, 256),
    # more maps than a matrix instruction has columns, heads and rows that fill no tile, blocks of maps that end inside a key head's or
    # a latent's, latents in slices with a short last one
    "one32": shape(1, 1, 1, 32, 96), "q32": shape(32, 1, 1, 64, 128), "q20": shape(20, 1, 1, 64, 320), "w640": shape(1, 1, 1, 64, 640),
    "h32": shape(20, 4, 2, 32, 640), "q18": shape(18, 1, 1, 128, 512), "q17": shape(17, 1, 1, 96, 1280), "k5": shape(15, 5, 1, 64, 512),
    "w672": shape(12, 3, 3, 64, 672), "h160": shape(24, 8, 2, 160, 544), "q40": shape(40, 8, 4, 128, 256), "h544": shape(2, 1, 1, 544, 544),
}


class MxCache:
    """Caller-owned 8-bit cache: contiguous (page 0) or pages dealt in random order with spare ones between; every byte
    starts as a NaN code with a scale of 2^100, so that a row that should not be read shows.  missing: (slot, page) without
    a page."""

    def __init__(self, sh, slots, max_seq, page=0, seed=0, missing=()):
        self.kw, self.cw = sh["n_kgroups"] * sh["head_dim"], sh["n_cgroups"] * sh["latent_dim"]
        self.page, self.slots, self.max_seq = page, slots, max_seq
        if page:
            assert max_seq % page == 0
            pps = max_seq // page
            perm = np.random.default_rng(seed).permutation(slots * pps + 3)
            self.table_np = perm[:slots * pps].reshape(slots, pps).astype(np.int32)
            for s, i in missing:
                self.table_np[s, i] = -1
            self.table, lead = torch.from_numpy(self.table_np).cuda(), (slots * pps + 3, page)
        else:
            self.table, lead = None, (slots, max_seq)
        def byte(width, fill):
            return torch.full((*lead, width), fill, dtype=torch.uint8, device="cuda")
        self.k, self.c = byte(self.kw, 0x7f), byte(self.cw, 0xff)
        self.ks, self.cs = byte(self.kw // BLOCK, 227), byte(self.cw // BLOCK, 227)
        self.seq_lens = torch.zeros(slots, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(slots, dtype=torch.int32, device="cuda")
        parts = (self.k, self.c, self.ks, self.cs, self.seq_lens, self.status)
        self.struct = B.make_paged_mx_cache(*parts, self.table) if page else B.make_mx_cache(*parts)

    def rows(self, slot, lo, hi):
        """pool row of rows lo .. hi-1"""
        r = np.arange(lo, hi)
        return self.table_np[slot][r // self.page].astype(np.int64) * self.page + r % self.page if self.page else r + slot * self.max_seq

    def host(self):
        return [t.view(-1, t.shape[-1]).cpu().numpy() for t in (self.k, self.c, self.ks, self.cs)]

    def fill(self, lens, rng, spread=2.0):
        """Random rows in front of every slot's end: codes of ordinary numbers under scales 2^-spread .. 2^spread."""
        host = self.host()
        at = np.concatenate([self.rows(slot, 0, n) for slot, n in enumerate(lens)])
        n = len(at)
        for codes, scale, w in ((host[0], host[2], self.kw), (host[1], host[3], self.cw)):
            q, sc = quantise(rng.standard_normal((n, w)) * np.repeat(2.0 ** rng.uniform(-spread, spread, (n, w // BLOCK)), BLOCK, axis=1))
            # codes of exact e4m3 numbers
            order = np.argsort(E4M3[:127])
            mag = order[np.searchsorted(E4M3[:127][order], np.abs(q))]
            codes[at], scale[at] = (mag + 128 * np.signbit(q)).astype(np.uint8), sc
        for t, h in zip((self.k, self.c, self.ks, self.cs), host):
            t.copy_(torch.from_numpy(h).view(t.shape))
        self.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        return self


def attention(sh, q: np.ndarray, k: np.ndarray, c: np.ndarray):
    """One sequence in float64: q [n_q*d_h], k [n, kw], c [n, cw] -> (L [n_q*d_l], sum_t p_t |c_t|, the largest
    scale * sum_j |q_j k_tj| of a map, broadcast over its latents)."""
    nq, nk, nc, dh, dl = (sh[n] for n in ("n_qgroups", "n_kgroups", "n_cgroups", "head_dim", "latent_dim"))
    out, mag, big = np.zeros((nq, dl)), np.zeros((nq, dl)), np.zeros((nq, dl))
    if k.shape[0]:
        for g in range(nq):
            kg, cg = k[:, g * nk // nq * dh:][:, :dh], c[:, g * nc // nq * dl:][:, :dl]
            qg = q[g * dh:(g + 1) * dh]
            s = kg @ qg / np.sqrt(dh)
            p = np.exp(s - s.max())
            p /= p.sum()
            out[g], mag[g] = p @ cg, p @ np.abs(cg)
            big[g] = (np.abs(kg) @ np.abs(qg)).max() / np.sqrt(dh)
    return out.reshape(-1), mag.reshape(-1), big.reshape(-1)


def attention_bound(dtype, sh, n, ref, mag, big):
    """Largest error of fp32 sums in any order.  A score is a sum of d_h products (a rounding each, at most 2^-24 of the sum
    of magnitudes), times the scale and log2(e) (two more, and the exponential's own); p moves by that much, top and bottom.
    The weighted sum has n terms (a rounding each) and is joined, rescaled and divided (64).  Weights may be taken in two
    16-bit parts where the result has 16 bits (2^-16).  Then the result is rounded once."""
    u = 2.0 ** -24
    rel = 2 * (sh["head_dim"] + 4) * u * big + (n + 64) * u + (2.0 ** -16 if dtype == "bf16" else 0.0)
    err = rel * mag
    return err + HALF_STEP[dtype] * (np.abs(ref) + err)
