"""Workloads of the operators over a whole key / value pool: attention of a prompt, a chunk or a single
token that also accumulates every slot's attention weight, eviction by that weight, attention of a tree of
drafted tokens, and the append of the accepted path.

With `own` false `run` computes an operator in its plain form, elementary torch operations in 32 bits; with
`own` true it makes the library's calls.
"""
import math

import numpy as np
import torch

own = False

_DT = {"f16": torch.float16, "f32": torch.float32}
_ctx = None


def _attention(name, B, H, group, d, n_q, N, dtype, ragged, mass=True):
    return dict(name=name, op="attention", B=B, H=H, group=group, d=d, n_q=n_q, N=N, N_cap=N + N // 16 + 5,
                dtype=dtype, ragged=ragged, mass=mass)


def _tree(name, B, H, group, d, n_q, N, dtype, ragged):
    return dict(name=name, op="tree", B=B, H=H, group=group, d=d, n_q=n_q, N=N, N_cap=N + 64, dtype=dtype, ragged=ragged)


def _evict(name, B, H, d, N, keep, recent, dtype, ragged):
    return dict(name=name, op="evict", B=B, H=H, d=d, N=N, N_cap=N + 33, keep=keep, recent=recent, dtype=dtype,
                ragged=ragged)


def _append(name, B, H, d, n_rows, most, N, dtype, path):
    return dict(name=name, op="append", B=B, H=H, d=d, n_rows=n_rows, most=most, N=N, N_cap=N + most + 7, dtype=dtype,
                path=path)


def listed():
    return [
        # a short prompt of a small float32 model: the smallest prompt, bound by launches and latency
        _attention("prompt_f32_512", 1, 4, 1, 64, 512, 512, "f32", False),
        # the prompt of the batched 2048-token workload, weights accumulated for a later eviction
        _attention("prompt_f16_2048", 8, 32, 1, 128, 2048, 2048, "f16", False),
        # one chunk of a long prompt over what is cached already, sequences of different lengths, grouped heads
        _attention("chunk_f16_9001", 4, 8, 4, 128, 317, 9001, "f16", True),
        # a single sequence decoding: one token over a short cache, the smallest call of a serving loop
        _attention("token_f16_777", 1, 32, 1, 128, 1, 777, "f16", False),
        # a batch decoding over 4096 cached tokens
        _attention("token_f16_4096", 16, 32, 1, 128, 1, 4096, "f16", False),
        # decoding over a long context
        _attention("token_f16_32768", 4, 40, 1, 128, 1, 32768, "f16", False),
        # verification of a small tree of drafted tokens, one sequence
        _tree("tree_f16_13", 1, 32, 1, 128, 13, 2048, "f16", False),
        # verification of a full tree for a batch of ragged sequences with grouped heads
        _tree("tree_f16_63", 8, 8, 4, 128, 63, 8191, "f16", True),
        # a decode step at the budget: one entry too many in every head
        _evict("evict_step_2048", 8, 32, 128, 2049, 2048, 1024, "f16", False),
        # the eviction after a prompt: 4096 entries down to a fifth
        _evict("evict_prompt_4096", 16, 32, 128, 4096, 819, 409, "f16", False),
        # the accepted path of a drafted tree joins the pool
        _append("append_path_63", 8, 32, 128, 63, 5, 2048, "f16", True),
        # the keys and values of a prompt's chunk join the pool
        _append("append_chunk_2048", 16, 32, 128, 2048, 2048, 2048, "f16", False),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "tree", "tree", "evict", "append"])
    d = rng.choice([64, 128, 128, 128, 256, 32])
    dtype = rng.choice(["f16", "f16", "f16", "f32"])
    ragged = rng.random() < 0.5
    size = (4 if dtype == "f32" else 2) * d
    while True:
        B, H, group = _spread(rng, 1, 16), _spread(rng, 1, 40), rng.choice([1, 1, 2, 4, 8])
        N = _spread(rng, 16, 32768)
        if op == "attention":
            n_q = 1 if rng.random() < 0.4 else _spread(rng, 2, N)
            # no more products, and no more bytes, than the largest listed ones
            if B * H * group * n_q * N * d > 8 * 32 * 2048 * 2048 * 128 // 2 or B * H * N * size > 4 * 40 * 32768 * 256:
                continue
            return _attention("", B, H, group, d, n_q, N, dtype, ragged, mass=rng.random() < 0.8)
        if op == "tree":
            n_q = _spread(rng, 1, 64)
            if B * H * group * n_q * N * d > 8 * 32 * 63 * 8191 * 128 or B * H * N * size > 8 * 32 * 8191 * 256:
                continue
            return _tree("", B, H, group, d, n_q, N, dtype, ragged)
        if B * H * N * size > 16 * 32 * 4096 * 256:
            continue
        if op == "evict":
            keep = N - 1 if rng.random() < 0.3 else _spread(rng, 8, N - 1)
            return _evict("", B, H, d, N, keep, keep // rng.choice([2, 3, 8]), dtype, ragged)
        path = rng.random() < 0.6
        n_rows = _spread(rng, 1, 64) if path else _spread(rng, 1, 4096)
        if B * H * n_rows * size > 16 * 32 * 2048 * 256:
            continue
        return _append("", B, H, d, n_rows, min(n_rows, rng.randint(1, 8)) if path else n_rows, N, dtype, path)


def _lengths(case):
    """Valid entries and query rows of every sequence (of the case alone): all, or down to a quarter of them."""
    B, N, n_q = case["B"], case["N"], case.get("n_q", 1)
    kv = [N] * B
    nq = [n_q] * B
    if case.get("ragged"):
        kv = [max(1, N - (3 * N // 4) * b // B) for b in range(B)]
        nq = [max(1, n_q - (n_q // 2) * b // B) for b in range(B)]
    return kv, nq


def _appended(case):
    return [1 + (case["most"] - 1) * (B_i + 1) // case["B"] for B_i in range(case["B"])] if case["path"] \
        else [case["n_rows"]] * case["B"]


def _tensor(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DT[case["dtype"]]
    B, H, d, N, N_cap = (case[k] for k in ("B", "H", "d", "N", "N_cap"))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=dt)

    kv, nq = _lengths(case)
    st = dict(case=case, K=normal(B, H, N_cap, d), V=normal(B, H, N_cap, d), kv_len=_tensor(kv))
    # a few heavy hitters in every sequence
    heavy = torch.randint(0, N, (B, max(1, N // 100)), generator=g, device="cuda")
    for b in range(B):
        st["K"][b, :, heavy[b]] *= 2
    if case["op"] in ("attention", "tree"):
        T, Hq = case["n_q"], H * case["group"]
        st["q"] = normal(B, T, Hq, d)
        st["q_len"] = _tensor(nq)
        st["scale"] = 2.0 / math.sqrt(d)
        st["out"] = torch.zeros((B, T, Hq, d), dtype=dt, device="cuda")
        if case["op"] == "attention":
            # what earlier steps have accumulated
            st["mass"] = torch.empty((B * H, N_cap), device="cuda").exponential_(1.0, generator=g) if case["mass"] else None
        else:
            st["k_tree"], st["v_tree"] = normal(B, T, H, d), normal(B, T, H, d)
            r = np.random.default_rng(seed)
            visible = np.zeros((B, T), np.uint64)
            for b in range(B):
                for i in range(T):
                    visible[b, i] = np.uint64(1) << np.uint64(i)
                    if i:          # a node's parent is one of the nodes before it, and mostly one of the first
                        visible[b, i] |= visible[b, int(r.integers(0, i) * r.random())]
            st["visible"] = torch.from_numpy(visible.view(np.int64)).cuda()
    elif case["op"] == "evict":
        mass = torch.empty((B * H, N_cap), device="cuda").exponential_(1.0, generator=g) ** 3
        mass[torch.rand((B * H, N_cap), generator=g, device="cuda") < 0.05] = 0.0      # never attended yet
        if case["keep"] == N - 1:          # a pool that has been evicted from before: any order of positions
            born = torch.argsort(torch.rand((B * H, N_cap), generator=g, device="cuda"), dim=1).int()
            born[:, N - 1] = N_cap
            st["protect_from"] = _tensor([N_cap - case["recent"]] * B)
        else:
            born = torch.arange(N_cap, device="cuda", dtype=torch.int32).repeat(B * H, 1)
            st["protect_from"] = st["kv_len"] - case["recent"]
        st["state"] = torch.stack([mass, born.view(torch.float32)])
    else:
        T = case["n_rows"]
        st["k_rows"], st["v_rows"] = normal(B, T, H, d), normal(B, T, H, d)
        st["n_append"] = _tensor(_appended(case))
        st["path"] = None
        if case["path"]:                   # ascending nodes of the tree
            p = torch.rand((B, T), generator=g, device="cuda").argsort(1)[:, :case["most"]].sort(1).values
            st["path"] = torch.cat([p, torch.zeros((B, T - case["most"]), dtype=p.dtype, device="cuda")], 1).int()
        st["pos"] = st["kv_len"] + 100
        st["mass"] = torch.empty((B * H, N_cap), device="cuda").exponential_(1.0, generator=g)
        st["born"] = torch.arange(N_cap, device="cuda", dtype=torch.int32).repeat(B * H, 1)
    if own:
        _prepare_own(st)
    return st


def _prepare_own(st):
    global _ctx
    import paper_2406_19707_amd as ig
    if _ctx is None:
        _ctx = ig.Context(0)
    c = st["case"]
    st["desc"] = ig.IgDesc(B=c["B"], H=c["H"], d=c["d"], r=1, N=c["N"], N_cap=c["N_cap"],
                           dtype=ig.IG_F32 if c["dtype"] == "f32" else ig.IG_F16, scale=st.get("scale", 1.0))
    if c["op"] in ("attention", "tree"):
        _ctx.ig_reserve_cache(st["desc"], c["group"], c["n_q"])
    elif c["op"] == "evict":
        _ctx.ig_reserve_cache(st["desc"], 1, 1)


def run(st):
    c = st["case"]
    if c["op"] == "attention":
        return _run_attention(st, c)
    if c["op"] == "tree":
        return _run_tree(st, c)
    if c["op"] == "evict":
        return _run_evict(st, c)
    return _run_append(st, c)


def _softmax_product(logits, V):
    """softmax of logits (-inf where nothing may be seen) times V, rows that see nothing zero; and the weights."""
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = (logits - top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    return p @ V, p


def _rows(q, H):
    """[B, T, H*G, d] -> float32 [B, H, T*G, d]"""
    B, T, Hq, d = q.shape
    return q.float().view(B, T, H, Hq // H, d).permute(0, 2, 1, 3, 4).reshape(B, H, -1, d)


def _heads(x, T, G):
    """[B, H, T*G, d] -> [B, T, H*G, d]"""
    B, H, _, d = x.shape
    return x.view(B, H, T, G, d).permute(0, 2, 1, 3, 4).reshape(B, T, H * G, d)


def _run_attention(st, c):
    B, H, G, T, N = c["B"], c["H"], c["group"], c["n_q"], c["N"]
    if own:
        _ctx.ig_cache_attention(st["desc"], G, T, st["q"], st["q_len"], st["K"], st["V"], st["kv_len"], st["mass"],
                                st["out"])
    else:
        K, V = st["K"][:, :, :N].float(), st["V"][:, :, :N].float()
        i = torch.arange(T, device="cuda")
        last = st["kv_len"][:, None] - st["q_len"][:, None] + i                        # [B, T]
        valid = i < st["q_len"][:, None]
        seen = (torch.arange(N, device="cuda") <= last[:, :, None]) & valid[:, :, None]
        seen = seen[:, None].repeat_interleave(G, 2)                                   # [B, 1, T*G, N]
        logits = (_rows(st["q"], H) @ K.transpose(2, 3)).mul_(st["scale"])
        logits.masked_fill_(~seen, -math.inf)
        out, p = _softmax_product(logits, V)
        st["out"].copy_(torch.where(valid[:, :, None, None], _heads(out, T, G), st["out"].float()))
        if st["mass"] is not None:
            st["mass"][:, :N] += p.sum(2).view(B * H, N)
    return dict(out=st["out"], mass=st["mass"]) if st["mass"] is not None else dict(out=st["out"])


def _run_tree(st, c):
    H, G, T, N = c["H"], c["group"], c["n_q"], c["N"]
    if own:
        _ctx.ig_tree_attention(st["desc"], G, T, st["q"], st["k_tree"], st["v_tree"], st["visible"], st["q_len"],
                               st["K"], st["V"], st["kv_len"], st["out"])
        return st["out"]
    K = torch.cat([st["K"][:, :, :N], st["k_tree"].transpose(1, 2)], 2).float()
    V = torch.cat([st["V"][:, :, :N], st["v_tree"].transpose(1, 2)], 2).float()
    i = torch.arange(T, device="cuda")
    valid = i < st["q_len"][:, None]                                                   # [B, T]
    seen = torch.cat([(torch.arange(N, device="cuda") < st["kv_len"][:, None])[:, None].expand(-1, T, -1),
                      ((st["visible"][:, :, None] >> i) & 1).bool() & valid[:, None]], 2) & valid[:, :, None]
    logits = (_rows(st["q"], H) @ K.transpose(2, 3)).mul_(st["scale"])
    logits.masked_fill_(~seen[:, None].repeat_interleave(G, 2), -math.inf)
    out, _ = _softmax_product(logits, V)
    st["out"].copy_(torch.where(valid[:, :, None, None], _heads(out, T, G), st["out"].float()))
    return st["out"]


def _run_evict(st, c):
    B, H, N, keep = c["B"], c["H"], c["N"], c["keep"]
    state = st["state"].clone()            # a pass starts from the same weights
    mass, born = state[0], state[1].view(torch.int32)
    if own:
        _ctx.ig_pool_evict(st["desc"], keep, st["kv_len"], mass, born, st["protect_from"], None, None, st["K"], st["V"])
        return dict(K=st["K"], V=st["V"], mass=mass, born=born)
    n = st["kv_len"].repeat_interleave(H)[:, None]
    slot = torch.arange(N, device="cuda")
    key = torch.where(born[:, :N] >= st["protect_from"].repeat_interleave(H)[:, None], math.inf, mass[:, :N])
    key = torch.where(slot < n, key, -math.inf)
    order = key.argsort(dim=1, descending=True, stable=True)
    stays = torch.zeros((B * H, N), dtype=torch.bool, device="cuda").scatter_(1, order[:, :keep], True)
    moves = stays & (slot >= keep) & (slot < n)
    holes = ~stays & (slot < keep) & (slot < n)
    # the j-th slot that moves fills the j-th hole: both lists in order of (pool, slot)
    pool, src = moves.nonzero(as_tuple=True)
    _, dst = holes.nonzero(as_tuple=True)
    for rows in (st["K"].view(B * H, -1, c["d"]), st["V"].view(B * H, -1, c["d"]), mass, born):
        rows[pool, dst] = rows[pool, src]
    return dict(K=st["K"], V=st["V"], mass=mass, born=born)


def _run_append(st, c):
    B, H, T, d = c["B"], c["H"], c["n_rows"], c["d"]
    if own:
        _ctx.ig_append_rows(st["desc"], T, st["k_rows"], st["v_rows"], st["path"], st["n_append"], st["kv_len"], st["pos"],
                            None, None, st["K"], st["V"], st["mass"], st["born"])
    else:
        j = torch.arange(T, device="cuda")
        b, j = (j < st["n_append"][:, None]).nonzero(as_tuple=True)
        slot = st["kv_len"][b] + j
        src = j if st["path"] is None else st["path"][b, j]
        st["K"][b, :, slot] = st["k_rows"][b, src]
        st["V"][b, :, slot] = st["v_rows"][b, src]
        st["mass"].view(B, H, -1)[b, :, slot] = 0.0
        st["born"].view(B, H, -1)[b, :, slot] = (st["pos"][b] + j)[:, None].int()
    return dict(K=st["K"], V=st["V"], mass=st["mass"], born=st["born"])


def _pairs(case):
    """Pairs of a query token and an entry it sees, over the batch (one head)."""
    kv, nq = _lengths(case)
    total = 0
    for n, m in zip(kv, nq):
        if case["op"] == "tree":
            total += m * n + m * (m + 1) // 2
        else:
            first = n - m + 1                  # entries the first query sees, may be below 1
            lo = max(first, 1)
            total += (lo + n) * (n - lo + 1) // 2 if n >= lo else 0
    return total


def work(case):
    B, H, d = case["B"], case["H"], case["d"]
    row = d * (4 if case["dtype"] == "f32" else 2)
    kv, nq = _lengths(case)
    if case["op"] in ("attention", "tree"):
        Hq = H * case["group"]
        nbytes = sum(kv) * H * 2 * row + sum(nq) * Hq * 2 * row
        if case["op"] == "tree":
            nbytes += sum(nq) * (H * 2 * row + 8)
        elif case["mass"]:
            nbytes += sum(kv) * H * 8
        return {"bytes": nbytes, "flops": 4 * d * Hq * _pairs(case)}
    if case["op"] == "evict":
        nbytes = 0
        for n in kv:
            out = max(0, n - case["keep"])
            # entries that move: those that stay among the last n - keep; the newest `recent` all stay, of the others
            # an even share (a pool in any order: of all)
            recent = min(case["recent"], case["keep"], n)
            if case["keep"] == case["N"] - 1:
                moved = out * case["keep"] / n
            else:
                old = n - recent
                tail = max(0, out - recent)
                moved = min(recent, out) + (tail * (case["keep"] - recent) / old if old else 0)
            nbytes += H * (n * 8 + moved * (2 * 2 * row + 16))
        return {"bytes": int(nbytes), "flops": 0}
    return {"bytes": sum(_appended(case)) * H * (4 * row + 8), "flops": 0}


def exact(case, seed):
    """What `run` returns, from the definitions: sequence by sequence and head by head, in 64 bits."""
    st = prepare_inputs(case, seed)
    kv, nq = _lengths(case)
    B, H, d = case["B"], case["H"], case["d"]
    if case["op"] in ("attention", "tree"):
        G, T = case["group"], case["n_q"]
        out = st["out"].double()
        mass = st["mass"].double() if st.get("mass") is not None else None
        for b in range(B):
            n, m = kv[b], nq[b]
            for h in range(H):
                K, V = st["K"][b, h, :n].double(), st["V"][b, h, :n].double()
                if case["op"] == "tree":
                    K = torch.cat([K, st["k_tree"][b, :m, h].double()])
                    V = torch.cat([V, st["v_tree"][b, :m, h].double()])
                    bits = [int(v) & (2 ** 64 - 1) for v in st["visible"][b, :m].tolist()] if h == 0 else None
                    if h == 0:
                        sees = torch.ones((m, n + m), dtype=torch.bool)
                        for i in range(m):
                            for j in range(m):
                                sees[i, n + j] = bool(bits[i] >> j & 1)
                        sees = sees.cuda()
                else:
                    sees = torch.ones((m, n), dtype=torch.bool, device="cuda").tril(n - m)
                for gq in range(h * G, h * G + G):
                    weight = torch.exp2(_log2_weights(st["q"][b, :m, gq].double() @ K.T * st["scale"], sees))
                    out[b, :m, gq] = weight @ V
                    if mass is not None:
                        mass[b * H + h, :n] += weight.sum(0)
        if case["op"] == "tree":
            return out
        return dict(out=out, mass=mass) if mass is not None else dict(out=out)
    K, V = st["K"].double(), st["V"].double()
    if case["op"] == "append":
        mass, born = st["mass"].double(), st["born"].clone()
        for b, count in enumerate(_appended(case)):
            rows = list(range(count)) if st["path"] is None else st["path"][b, :count].tolist()
            n = kv[b]
            K[b, :, n:n + count] = st["k_rows"][b, rows].double().transpose(0, 1)
            V[b, :, n:n + count] = st["v_rows"][b, rows].double().transpose(0, 1)
            mass[b * H:b * H + H, n:n + count] = 0
            born[b * H:b * H + H, n:n + count] = int(st["pos"][b]) + torch.arange(count, device="cuda", dtype=torch.int32)
        return dict(K=K, V=V, mass=mass, born=born)
    mass = st["state"][0].double().cpu().numpy()
    born = st["state"][1].view(torch.int32).cpu().numpy().copy()
    keep, limit = case["keep"], st["protect_from"].tolist()
    for i in range(B * H):
        n = kv[i // H]
        if n <= keep:
            continue
        safe = born[i, :n] >= limit[i // H]
        # by protection, then weight, then slot: the last key of lexsort counts most
        rank = np.lexsort((np.arange(n), -mass[i, :n], ~safe))
        stay = np.sort(rank[:keep])
        src = stay[stay >= keep]
        dst = np.setdiff1d(np.arange(keep), stay)
        K[i // H, i % H, dst] = K[i // H, i % H, src]
        V[i // H, i % H, dst] = V[i // H, i % H, src]
        mass[i, dst], born[i, dst] = mass[i, src], born[i, src]
    return dict(K=K, V=V, mass=torch.from_numpy(mass).cuda(), born=torch.from_numpy(born).cuda())


def _log2_weights(logits, sees):
    """Base-2 logarithm of the softmax weights of 64-bit logits; -inf where nothing is seen."""
    t = torch.where(sees, logits * math.log2(math.e), -math.inf)
    return torch.where(sees, t - torch.logsumexp(t * math.log(2.0), 1, keepdim=True) / math.log(2.0), -math.inf)


def prepare_inputs(case, seed):
    """The inputs alone, without the library's descriptor."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was
