"""Shared plumbing of the tests of pages of 8-bit codes: inputs, the definitions in 64 bits, and tolerances."""
from __future__ import annotations

import math

import numpy as np
import torch

import paper_2406_19707_amd as ig
from ig_cache import DT, SENTINEL, definition, desc, i32, rows, weight_error  # noqa: F401

CODES = {"i8": ig.IG_CODE_I8, "e4m3": ig.IG_CODE_E4M3}
KIND = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}
MOST = {"i8": 127.0, "e4m3": 448.0}
LEAST = 2.0 ** -80
JUNK = {"i8": 0x55, "e4m3": 0x7F}               # a code that shows (e4m3: NaN)


class Pages:
    """A pool of pages for B sequences of up to N_cap slots, pages in any order; everything in it is junk but what `fill` writes."""

    def __init__(self, B, H, d, N_cap, page, code, seed=0, spare=2):
        g = torch.Generator().manual_seed(seed)
        per = -(-N_cap // page)
        n = B * per + spare
        self.shape, self.code, self.page = (B, H, d, N_cap), code, page
        self.table = torch.randperm(n, generator=g)[:B * per].view(B, per).int().cuda()
        self.K, self.V = (torch.full((n, H, page, d), JUNK[code], dtype=torch.uint8, device="cuda") for _ in "KV")
        self.K_scale, self.V_scale = (torch.full((n, H), float("nan"), device="cuda") for _ in "KV")

    def struct(self, **changed):
        p = ig.IgPages(self.table, self.K, self.V, self.K_scale, self.V_scale, CODES[self.code])
        for k, v in changed.items():
            setattr(p, k, v)
        return p

    def fill(self, kv, seed, spread=3):
        """Random codes in the first kv[b] slots of every sequence, scales of 2^-spread .. 2^spread around one that makes values
        of about 1."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        B, H, d, _ = self.shape
        for b, n in enumerate(kv):
            for c in range(-(-n // self.page)):
                at, m = int(self.table[b, c]), min(self.page, n - c * self.page)
                for x, s in ((self.K, self.K_scale), (self.V, self.V_scale)):
                    v = torch.randn((H, m, d), generator=g, device="cuda") * (30 if self.code == "i8" else 110)
                    v = v.clamp(-MOST[self.code], MOST[self.code])
                    x[at, :, :m] = (v.round().to(torch.int8) if self.code == "i8" else v.to(torch.float8_e4m3fn)).view(torch.uint8)
                    e = torch.randint(-spread, spread + 1, (H,), generator=g, device="cuda") - (5 if self.code == "i8" else 7)
                    s[at] = torch.exp2(e.float())
        return self

    def values(self, x, b, n):
        """The first n slots of sequence b in 64 bits: [H, n, d]"""
        B, H, d, _ = self.shape
        codes, scale = getattr(self, x), getattr(self, x + "_scale")
        at = self.table[b, :-(-n // self.page)].long()
        v = codes[at].view(KIND[self.code]).double() * scale[at].double()[:, :, None, None]
        return v.transpose(0, 1).reshape(H, -1, d)[:, :n]

    def state(self):
        return [t.clone() for t in (self.K, self.V, self.K_scale.view(torch.int32), self.V_scale.view(torch.int32))]


def out_tolerance(dtype, ref, absum, size, n, d, biggest, vscales):
    """Absolute error of an output row.  Its own rounding; the weights' error in float32, in which the logit also meets the
    exponent of its page's scale (at most 80 beside `size`: half a step of that, twice); the sum's roundings; and the weights, times their
    page's scale, as halves: half a step of 2^-10, or of 2^-24 below the normal range, where the largest is at least 2^8 (float32:
    two halves, 2^-22 and the same below).  biggest: a code's largest value times the largest scale.  Float32 queries as two halves: 2^-22
    of themselves, i.e. of `size`, and 2^-38 of the row's largest, at most d times that of `size` in all."""
    e = weight_error(size, n, d) + n * 2.0 ** -24 + 2 * vscales * 2.0 ** -24
    if dtype == "f32":
        e = e + 2 * (2.0 ** -22 + d * 2.0 ** -38) * size
        return 2.0 ** -24 * ref.abs() + (e + 2.0 ** -22) * absum + n * 2.0 ** -33 * biggest + 2.0 ** -126
    return 2.0 ** -11 * ref.abs() + (e + 2.0 ** -11) * absum + n * 2.0 ** -33 * biggest + 2.0 ** -25


def check_attention(pages, q, kv, nq, group, scale, dtype, out, before):
    B, H, d, _ = pages.shape
    for b in range(B):
        n, m = kv[b], nq[b]
        assert torch.equal(out[b, m:], before[b, m:]), f"rows from {m} of sequence {b} were written"
        if m == 0:
            continue
        K, V = (pages.values(x, b, n) for x in "KV")
        sees = torch.arange(n, device="cuda") <= (n - m + torch.arange(m, device="cuda"))[:, None]
        used = pages.V_scale[pages.table[b, :-(-n // pages.page)].long()] if n else torch.ones((1, H), device="cuda")
        for h in range(H):
            biggest = used[:, h].max().item() * MOST[pages.code]
            spread = used[:, h].log2().abs().max().item()
            for g in range(group):
                ref, p, absum, size = definition(q[b, :m, h * group + g], K[h], V[h], sees, scale)
                tol = out_tolerance(dtype, ref, absum, size, n, d, biggest, spread)
                got = out[b, :m, h * group + g].double()
                bad = ~((got - ref).abs() <= tol)
                assert not bad.any(), (f"sequence {b} head {h * group + g}: error {((got - ref).abs() / tol).max().item():.2f} "
                                       f"tolerances at row {bad.any(1).nonzero()[0].item()}")


def run_attention(ctx, dtype, code, d, B, H, group, n_q, N, N_cap, page, kv=None, nq=None, scale=None, seed=0, stream=None, spread=3):
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    lens, qlens = kv or [N] * B, nq or [n_q] * B
    pages = Pages(B, H, d, N_cap, page, code, seed).fill(lens, seed + 1, spread)
    q = rows((B, n_q, H * group, d), dtype, seed + 2)
    for b, m in enumerate(qlens):
        q[b, m:] = float("nan")
    out = torch.full_like(q, SENTINEL)
    before = out.clone()
    ctx.ig_page_attention(desc(B, H, d, N, N_cap, dtype, scale), pages.struct(), group, n_q, q, i32(nq), i32(kv), out, stream)
    torch.cuda.synchronize()
    check_attention(pages, q, lens, qlens, group, float(np.float32(scale)), dtype, out, before)
    return out


# ---- rotation and append -----------------------------------------------------------------------------------------------

def rotary(dims, interleaved=False, kind=ig.IG_ROPE_PLAIN, **more):
    freq, magnitude = ig.ig_rotary_frequencies(dims, kind=kind, **more)
    return ig.IgRotary(torch.from_numpy(freq).cuda(), dims=dims, interleaved=interleaved, magnitude=magnitude), freq, magnitude


def turned(x, pos, dims, interleaved, freq, magnitude, inverse=False):
    """x [n, heads, d] rotated in 64 bits, and the bound that a rotation's rounding is measured by: |a| + |b| of each pair"""
    x, out = x.double(), x.double().clone()
    size = torch.zeros_like(x)
    angle = pos.double()[:, None, None] * torch.from_numpy(freq).to(x.device)
    cos, sin = angle.cos() * magnitude, angle.sin() * magnitude * (-1 if inverse else 1)
    a = slice(0, dims, 2) if interleaved else slice(0, dims // 2)
    b = slice(1, dims, 2) if interleaved else slice(dims // 2, dims)
    out[..., a], out[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    size[..., a] = size[..., b] = (x[..., a].abs() + x[..., b].abs()) * abs(magnitude)
    return out, size


# A rotated value in float32: the angle's product in double (2^-53 of at most 2^31 turns' angle: 2^-22 of a radian at 2^31, 2^-36 at 2^17) is
# exact to the float32 it is reduced to (half a step of at most pi/4); sine and cosine by polynomials of 7 steps on at most 1, each half a
# step, and their last product with the magnitude; two products and their sum.  In half steps of 2^-23: 1 (reduction) + 7 + 2 + 2 = 12.
ROTATION = 12 * 2.0 ** -24


def needed_exponent(top, code):
    """The least e >= -80 with top <= most * 2^e"""
    e = -80
    if top > 0:
        e = max(e, math.frexp(top / MOST[code])[1] - 1)
        while top > MOST[code] * 2.0 ** e:
            e += 1
    return e
