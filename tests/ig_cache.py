"""Shared plumbing of the tests of attention over a whole pool: inputs, the definition in 64 bits, and tolerances."""
from __future__ import annotations

import numpy as np
import torch

import paper_2406_19707_amd as ig

DT = {"f16": torch.float16, "f32": torch.float32}
SENTINEL = 7.25


def desc(B, H, d, N, N_cap, dtype, scale=1.0, r=1):
    return ig.IgDesc(B=B, H=H, d=d, r=r, N=N, N_cap=N_cap, dtype=ig.IG_F32 if dtype == "f32" else ig.IG_F16, scale=scale)


def i32(values):
    return None if values is None else torch.tensor(values, dtype=torch.int32, device="cuda")


def pools(B, H, d, N_cap, dtype, kv, seed, junk=(float("nan"), float("inf"))):
    """K, V [B,H,N_cap,d]; what lies behind a sequence's valid slots is not finite."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    K = torch.randn((B, H, N_cap, d), generator=g, device="cuda").to(DT[dtype])
    V = torch.randn((B, H, N_cap, d), generator=g, device="cuda").to(DT[dtype])
    for b, n in enumerate(kv):
        K[b, :, n:], V[b, :, n:] = junk
    return K, V


def rows(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(DT[dtype])


def definition(q, K, V, sees, scale):
    """One (sequence, pool head): q [m, d], K, V [n, d] and sees [m, n] in 64 bits -> out, weights, and the two
    bounds the tolerances are made of: sum of |p v| and the largest scale * |q| . |k| of each row."""
    q, K, V = q.double(), K.double(), V.double()
    if K.shape[0] == 0:
        z = torch.zeros_like(q)
        return z, torch.zeros((q.shape[0], 0), dtype=torch.float64, device=q.device), z, torch.zeros_like(q[:, :1])
    s = torch.where(sees, q @ K.T * scale, -torch.inf)
    top = s.amax(1, keepdim=True)
    p = torch.exp(s - torch.where(top == -torch.inf, 0.0, top))
    l = p.sum(1, keepdim=True)
    p = p / torch.where(l == 0, 1.0, l)
    size = torch.where(sees, q.abs() @ K.abs().T * abs(scale), 0.0).amax(1, keepdim=True)
    return p @ V, p, p @ V.abs(), size


def weight_error(size, n, d):
    """Relative error of a weight in float32.  The logit is a float32 sum of d products (at most d roundings, of at
    most `size` each time), then scaled by a rounded constant and subtracted from its rounded maximum (3 more, the
    maximum's being as large): d + 4 half steps of 2^-24 of `size`, twice because the maximum has them too, times
    ln 2 over ln 2.  The exponential is good to 2^-22; the sum of n of them adds n half steps, the division and the
    joins of partial sums at most 8."""
    return 2 * (d + 4) * 2.0 ** -24 * size + 2.0 ** -22 + (n + 8) * 2.0 ** -24


def out_tolerance(dtype, ref, absum, size, n, d, V):
    """Absolute error of an output row: its own rounding, the weights' error, the sum's n roundings, and in half
    precision the weights' rounding to it (half a step of 2^-10, or of 2^-24 below its normal range, where the
    weights are relative to the largest)."""
    e = weight_error(size, n, d) + n * 2.0 ** -24
    if dtype == "f32":
        return 2.0 ** -24 * ref.abs() + e * absum + 2.0 ** -126
    vmax = V.double().abs().amax() if V.numel() else 0.0
    return 2.0 ** -11 * ref.abs() + (e + 2.0 ** -11) * absum + n * 2.0 ** -25 * vmax + 2.0 ** -25


def check_attention(q, K, V, kv, nq, group, scale, dtype, out, before, mass=None, mass0=None, tree=None):
    """out, mass of a call against the definition; rows and slots that the call leaves alone, bit for bit.
    tree: (k_tree, v_tree, visible as a list of lists of Python integers)"""
    B, H, _, d = K.shape
    for b in range(B):
        n, m = kv[b], nq[b]
        assert torch.equal(out[b, m:], before[b, m:]), f"rows from {m} of sequence {b} were written"
        for h in range(H):
            Kb, Vb = K[b, h, :n], V[b, h, :n]
            if tree is None:
                i = torch.arange(m, device="cuda")
                sees = torch.arange(n, device="cuda") <= (n - m + i)[:, None]
            else:
                Kb, Vb = torch.cat([Kb, tree[0][b, :m, h]]), torch.cat([Vb, tree[1][b, :m, h]])
                bits = torch.tensor([[v >> j & 1 for j in range(m)] for v in tree[2][b][:m]], dtype=torch.bool, device="cuda")
                sees = torch.cat([torch.ones((m, n), dtype=torch.bool, device="cuda"), bits.view(m, m)], 1)
            total = torch.zeros(n, dtype=torch.float64, device="cuda")
            slack = torch.zeros(n, dtype=torch.float64, device="cuda")
            for g in range(group):
                ref, p, absum, size = definition(q[b, :m, h * group + g], Kb, Vb, sees, scale)
                got = out[b, :m, h * group + g].double()
                tol = out_tolerance(dtype, ref, absum, size, Kb.shape[0], d, Vb)
                bad = ~((got - ref).abs() <= tol)
                assert not bad.any(), (f"sequence {b} head {h * group + g}: error {((got - ref).abs() / tol).max().item():.2f} "
                                       f"tolerances at row {bad.any(1).nonzero()[0].item()}")
                if mass is not None:
                    total += p.sum(0)
                    slack += (p * weight_error(size, n, d)).sum(0)
            if mass is not None:
                at = b * H + h
                assert torch.equal(mass[at, n:], mass0[at, n:]), "a slot behind the valid ones got a weight"
                ref = mass0[at, :n].double() + total
                # (m * group terms and the sum so far, each rounded once)
                tol = slack + (m * group + 4) * 2.0 ** -24 * (total + mass0[at, :n].double().abs()) + 2.0 ** -126
                err = (mass[at, :n].double() - ref).abs()
                assert (err <= tol).all(), f"pool {at}: weight off by {(err / tol).max().item():.2f} tolerances"


def run_attention(ctx, dtype, d, B, H, group, n_q, N, N_cap, kv, nq, with_mass=True, scale=None, seed=0, stream=None):
    scale = 1.5 / np.sqrt(d) if scale is None else scale
    lens, qlens = kv or [N] * B, nq or [n_q] * B
    K, V = pools(B, H, d, N_cap, dtype, lens, seed)
    q = rows((B, n_q, H * group, d), dtype, seed + 1)
    for b, m in enumerate(qlens):
        q[b, m:] = float("nan")
    out = torch.full_like(q, SENTINEL)
    before = out.clone()
    mass = mass0 = None
    if with_mass:
        mass0 = torch.rand((B * H, N_cap), device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed + 2))
        mass = mass0.clone()
    ds = desc(B, H, d, N, N_cap, dtype, scale)
    ctx.ig_cache_attention(ds, group, n_q, q, i32(nq), K, V, i32(kv), mass, out, stream)
    torch.cuda.synchronize()
    check_attention(q, K, V, lens, qlens, group, float(np.float32(scale)), dtype, out, before, mass, mass0)
    return out


def run_tree(ctx, dtype, d, B, H, group, T, N, N_cap, kv, nt, visible, scale=None, seed=0, bad_nodes=()):
    scale = 1.5 / np.sqrt(d) if scale is None else scale
    lens, tlens = kv or [N] * B, nt or [T] * B
    K, V = pools(B, H, d, max(N_cap, 1), dtype, lens, seed)
    q, kt, vt = (rows((B, T, x, d), dtype, seed + 1 + x) for x in (H * group, H, H))
    for b, m in enumerate(tlens):
        q[b, m:], kt[b, m:], vt[b, m:] = float("nan"), float("nan"), float("inf")
    clean = kt.clone(), vt.clone()
    for j in bad_nodes:
        kt[:, j], vt[:, j] = float("inf"), float("nan")
    out = torch.full_like(q, SENTINEL)
    before = out.clone()
    bits = torch.from_numpy(np.array(visible, np.uint64).view(np.int64)).cuda()
    ctx.ig_tree_attention(desc(B, H, d, N, N_cap, dtype, scale), group, T, q, kt, vt, bits, i32(nt), K, V, i32(kv), out)
    torch.cuda.synchronize()
    check_attention(q, K, V, lens, tlens, group, float(np.float32(scale)), dtype, out, before, tree=(*clean, visible))


def random_tree(T, seed):
    """visible masks of a random tree: a node sees itself and its ancestors"""
    r = np.random.default_rng(seed)
    out = []
    for i in range(T):
        out.append(1 << i | (out[int(r.integers(0, i))] if i else 0))
    return out
