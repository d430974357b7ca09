"""Workloads of the operators over a key / value cache held in 8 bits: the rotary embedding of queries and keys on the
device, the append of rotated rows to pages of 8-bit codes with a scale for each page and head, the attention that reads
such pages, and rows read back out of them.

With `own` false `run` computes an operator in its plain form, elementary torch operations in 32 bits (angles in 64); with
`own` true it makes the library's calls.
"""
import math

import torch

own = False

_DT = {"f16": torch.float16, "f32": torch.float32}
_MOST = {"i8": 127.0, "e4m3": 448.0}             # the largest code
_LEAST = 2.0 ** -80                              # the smallest scale
_ctx = None


def _rotate(name, B, n, heads, d, dims, interleaved, scaling, inverse, dtype):
    return dict(name=name, op="rotate", B=B, n=n, heads=heads, d=d, dims=dims, interleaved=interleaved, scaling=scaling,
                inverse=inverse, dtype=dtype)


def _append(name, B, H, group, d, n_rows, N, page, code, dims, interleaved, dtype, ragged, fused):
    return dict(name=name, op="append", B=B, H=H, group=group, d=d, n_rows=n_rows, N=N, page=page, code=code, dims=dims,
                interleaved=interleaved, dtype=dtype, ragged=ragged, fused=fused)


def _attention(name, B, H, group, d, n_q, N, page, code, dtype, ragged):
    return dict(name=name, op="attention", B=B, H=H, group=group, d=d, n_q=n_q, N=N, page=page, code=code, dtype=dtype,
                ragged=ragged)


def _gather(name, B, H, d, N, rows, page, code, dtype):
    return dict(name=name, op="gather", B=B, H=H, d=d, N=N, rows=rows, page=page, code=code, dtype=dtype)


def listed():
    return [
        # the query of one decode step of a small float32 model: the smallest call, all of it latency
        _rotate("rotate_f32_1", 1, 1, 4, 64, 64, False, "plain", False, "f32"),
        # the queries of the batched 2048-token prompts, frequencies stretched for a longer context
        _rotate("rotate_f16_2048", 16, 2048, 32, 128, 128, False, "wavelength", False, "f16"),
        # a decode step of a batch: one row a sequence joins the pages, and its query heads are rotated with it
        _append("append_step_i8", 16, 8, 4, 128, 1, 4096, 32, "i8", 128, False, "f16", True, True),
        # a prompt's keys and values join empty pages
        _append("append_prompt_e4m3", 16, 32, 1, 128, 2048, 0, 64, "e4m3", 128, False, "f16", False, False),
        # a chunk of ragged float32 sequences that begins in the middle of a page; a quarter of the head rotated
        _append("append_chunk_f32", 3, 12, 1, 64, 317, 1000, 16, "i8", 16, True, "f32", True, False),
        # a single sequence decoding over a short cache, the smallest call of a serving loop
        _attention("token_i8_777", 1, 32, 1, 128, 1, 777, 32, "i8", "f16", False),
        # a batch decoding over 4096 cached tokens
        _attention("token_i8_4096", 16, 32, 1, 128, 1, 4096, 32, "i8", "f16", False),
        # ragged sequences decoding over a long context, grouped heads
        _attention("token_e4m3_32768", 16, 8, 4, 128, 1, 32768, 64, "e4m3", "f16", True),
        # one chunk of a long prompt over what is cached already, grouped heads, small pages
        _attention("chunk_i8_9001", 4, 8, 4, 128, 317, 9001, 16, "i8", "f16", True),
        # the prompt of the batched 2048-token workload
        _attention("prompt_i8_2048", 8, 32, 1, 128, 2048, 2048, 64, "i8", "f16", False),
        # the speculated rows of one layer, a twentieth of 2048 tokens in every head
        _gather("gather_i8_2048", 8, 32, 128, 2048, 102, 32, "i8", "f16"),
        # the same out of a long context
        _gather("gather_e4m3_32768", 4, 40, 128, 32768, 1638, 64, "e4m3", "f16"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _rotated(rng, d):
    """Rotated channels of a head of d."""
    return rng.choice([d, d, d // 2, max(2, d // 4 // 2 * 2)])


def draw(rng):
    op = rng.choice(["rotate", "append", "append", "attention", "attention", "attention", "gather"])
    dtype = rng.choice(["f16", "f16", "f16", "f32"])
    size = 4 if dtype == "f32" else 2
    code = rng.choice(["i8", "e4m3"])
    page = rng.choice([16, 32, 64, 128])
    d = rng.choice([64, 128, 128, 128, 256, 32])
    ragged = rng.random() < 0.5
    while True:
        if op == "rotate":
            d = rng.choice([32, 64, 80, 96, 128, 128, 256])
            B, n, heads = _spread(rng, 1, 16), _spread(rng, 1, 4096), _spread(rng, 1, 64)
            if B * n * heads * d * size > 16 * 2048 * 32 * 128 * 2:
                continue
            return _rotate("", B, n, heads, d, _rotated(rng, d), rng.random() < 0.4,
                           rng.choice(["plain", "linear", "ntk", "ramp", "wavelength"]), rng.random() < 0.3, dtype)
        B, H, group = _spread(rng, 1, 16), _spread(rng, 1, 40), rng.choice([1, 1, 2, 4, 8])
        N = _spread(rng, 16, 32768)
        if op == "append":
            n_rows = rng.choice([1, _spread(rng, 1, 4096)])
            N = rng.choice([0, N])
            # no more values, and no more pages before them, than the largest listed ones
            if B * n_rows * H * (group + 2) * d * size > 16 * 2048 * 32 * 3 * 128 * 2 or B * H * N * d > 16 * 8 * 32768 * 128:
                continue
            return _append("", B, H, group, d, n_rows, N, page, code, _rotated(rng, d), rng.random() < 0.4, dtype, ragged,
                           rng.random() < 0.5)
        if B * H * N * d > 16 * 8 * 32768 * 128:
            continue
        if op == "attention":
            n_q = 1 if rng.random() < 0.4 else _spread(rng, 2, N)
            if B * H * group * n_q * N * d > 8 * 32 * 2048 * 2048 * 128 // (4 if dtype == "f32" else 2):
                continue
            return _attention("", B, H, group, d, n_q, N, page, code, dtype, ragged)
        rows = _spread(rng, 1, N)
        if B * H * rows * d * size > 4 * 40 * 1638 * 128 * 2:
            continue
        return _gather("", B, H, d, N, rows, page, code, dtype)


def _lengths(case):
    """Valid slots, and query tokens or rows to append, of every sequence: all, or down to a quarter and a half of them."""
    B, N, n = case["B"], case["N"], case.get("n_q", case.get("n_rows", 1))
    kv, rows = [N] * B, [n] * B
    if case.get("ragged"):
        kv = [N and max(1, N - (3 * N // 4) * b // B) for b in range(B)]
        rows = [max(1, n - (n // 2) * b // B) for b in range(B)]
    return kv, rows


def _capacity(case):
    """Slots that a sequence's row of the page table holds."""
    most = case["N"] + case.get("n_rows", 0)
    return (most + case["page"] - 1) // case["page"] * case["page"]


_ORIGINAL = 2048          # the context that stretched frequencies come from


def _stretch(case):
    """Arguments of the frequencies: kind, factor, low, high"""
    return {"plain": (0, 1.0, 1.0, 1.0), "linear": (1, 4.0, 1.0, 1.0), "ntk": (2, 4.0, 1.0, 1.0), "ramp": (3, 8.0, 1.0, 32.0),
            "wavelength": (4, 8.0, 1.0, 4.0)}[case.get("scaling", "plain")]


def _frequencies(case):
    """Angles of one position, in 64 bits, and the factor of the rotated channels."""
    dims = case["dims"]
    kind, factor, low, high = _stretch(case)
    c = torch.arange(dims // 2, dtype=torch.float64)
    theta = 10000.0
    if kind == 2 and dims > 2:
        theta *= factor ** (dims / (dims - 2))
    f = theta ** (-2 * c / dims)
    if kind == 1:
        f = f / factor
    if kind == 3:
        # the pair that turns n times over the original context
        at = [dims * math.log(_ORIGINAL / (2 * math.pi * n)) / (2 * math.log(theta)) for n in (high, low)]
        first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), dims - 1)
        r = ((c - first) / max(last - first, 0.001)).clamp(0, 1)
        f = f * (1 - r) + f / factor * r
    if kind == 4:
        s = ((_ORIGINAL * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        f = f * s + f / factor * (1 - s)
    return f, 0.1 * math.log(factor) + 1 if kind == 3 else 1.0


def _tensor(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _codes(shape, code, g):
    """Codes as rounding to a block's largest value leaves them, as bytes"""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float16)
    if code == "i8":
        return x.mul_(28).round_().clamp_(-127, 127).to(torch.int8).view(torch.uint8)
    return x.mul_(100).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DT[case["dtype"]]
    d, B = case["d"], case["B"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=dt)

    st = dict(case=case)
    if case["op"] == "rotate":
        n = case["n"]
        st["x"] = normal(B * n, case["heads"], d)
        # sequences that begin anywhere up to a long context
        begin = torch.randint(0, 1 << 17, (B, 1), generator=g, device="cuda")
        st["pos"] = (begin + torch.arange(n, device="cuda")).view(-1).int()
        st["out"] = torch.zeros_like(st["x"])
    else:
        H, page, code = case["H"], case["page"], case["code"]
        kv, rows = _lengths(case)
        per = _capacity(case) // page
        n_pages = B * per + 3
        # a pool of pages in any order, as one that has served for some time
        st["table"] = torch.randperm(n_pages, generator=g, device="cuda")[:B * per].view(B, per).int()
        st["kv_len"] = _tensor(kv)
        for x in "KV":
            st[x] = _codes((n_pages, H, page, d), code, g)
            spread = torch.randint(-2, 1, (n_pages, H), generator=g, device="cuda").float()
            st[x + "_scale"] = torch.exp2(spread - (4 if code == "i8" else 6))
        if case["op"] == "attention":
            T, Hq = case["n_q"], H * case["group"]
            st["q"], st["q_len"] = normal(B, T, Hq, d), _tensor(rows)
            st["scale"] = 2.0 / math.sqrt(d)
            st["out"] = torch.zeros((B, T, Hq, d), dtype=dt, device="cuda")
        elif case["op"] == "append":
            T, Hq = case["n_rows"], H * case["group"]
            # the projections' outputs, of a model with a few strong channels; one buffer for all three, or one each
            strong = torch.ones(d, device="cuda", dtype=dt)
            strong[torch.randint(0, d, (max(1, d // 16),), generator=g, device="cuda")] = 5
            if case["fused"]:
                st["qkv"] = normal(B, T, Hq + 2 * H, d) * strong
                st["q"], st["k"], st["v"] = st["qkv"].split([Hq, H, H], 2)
            else:
                st["q"], st["k"], st["v"] = (normal(B, T, h, d) * strong for h in (Hq, H, H))
            st["n_append"], st["q_out"] = _tensor(rows), torch.zeros((B, T, Hq, d), dtype=dt, device="cuda")
            st["pos"] = st["kv_len"] + 100
            # the slots of every page that gets a row: its values are read back
            slots = torch.arange((T + 2 * page - 2) // page * page, device="cuda", dtype=torch.int32)
            st["sel_idx"] = (st["kv_len"][:, None] // page * page + slots).clamp_(max=_capacity(case) - 1)[:, None].expand(-1, H, -1) \
                .reshape(B * H, -1).contiguous()
            st["sel_cnt"] = (st["kv_len"] % page + st["n_append"]).int()[:, None].expand(-1, H).reshape(-1).contiguous()
        else:
            pick = torch.rand((B * H, case["N"]), generator=g, device="cuda").argsort(1)[:, :case["rows"]]
            st["sel_idx"] = pick.sort(1).values.int().contiguous()
            least = max(1, case["rows"] * 3 // 4)
            st["sel_cnt"] = torch.randint(least, case["rows"] + 1, (B * H,), generator=g, device="cuda").int()
        if "sel_idx" in st:
            # (values of up to 8 significant bits: half precision holds them)
            kept = torch.float16 if case["op"] == "append" else dt
            for x in ("K_sel", "V_sel"):
                st[x] = torch.zeros((B * H, st["sel_idx"].shape[1], d), dtype=kept, device="cuda")
    if own:
        _prepare_own(st)
    return st


def _prepare_own(st):
    global _ctx
    import paper_2406_19707_amd as ig
    if _ctx is None:
        _ctx = ig.Context(0)
    c = st["case"]
    if "dims" in c:
        kind, factor, low, high = _stretch(c)
        freq, magnitude = ig.ig_rotary_frequencies(c["dims"], 10000.0, kind if c["dims"] > 2 else 0 if kind == 2 else kind, factor, low,
                                                   high, _ORIGINAL)
        st["freq"] = torch.from_numpy(freq).cuda()
        st["rotary"] = ig.IgRotary(st["freq"], dims=c["dims"], interleaved=c["interleaved"], magnitude=magnitude)
    st["dtype"] = ig.IG_F32 if c["dtype"] == "f32" else ig.IG_F16
    if c["op"] == "rotate":
        return
    code = ig.IG_CODE_I8 if c["code"] == "i8" else ig.IG_CODE_E4M3
    st["pages"] = ig.IgPages(st["table"], st["K"], st["V"], st["K_scale"], st["V_scale"], code)

    def desc(dtype):
        return ig.IgDesc(B=c["B"], H=c["H"], d=c["d"], r=1, N=c["N"], N_cap=_capacity(c), dtype=dtype, scale=st.get("scale", 1.0))

    st["desc"] = desc(st["dtype"])
    st["read"] = desc(ig.IG_F16) if c["op"] == "append" else st["desc"]
    if c["op"] == "attention":
        _ctx.ig_reserve_pages(st["desc"], c["group"], c["n_q"])


def run(st):
    return {"rotate": _run_rotate, "append": _run_append, "attention": _run_attention, "gather": _run_gather}[st["case"]["op"]](st, st["case"])


def _turn(x, pos, c):
    """x [n, heads, d] rotated at pos [n], in 32 bits"""
    f, magnitude = _frequencies(c)
    angle = pos.double()[:, None] * f.to(x.device)
    cos, sin = (angle.cos() * magnitude).float()[:, None], (angle.sin() * magnitude).float()[:, None]
    if c.get("inverse"):
        sin = -sin
    x, dims = x.float(), c["dims"]
    if c["interleaved"]:
        a, b = x[..., :dims:2], x[..., 1:dims:2]
        return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., dims:]], -1)
    a, b = x[..., :dims // 2], x[..., dims // 2:dims]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., dims:]], -1)


def _run_rotate(st, c):
    if own:
        _ctx.ig_rotate_rows(st["dtype"], c["B"] * c["n"], c["heads"], c["d"], st["rotary"], int(c["inverse"]), st["pos"], st["x"], 0,
                            st["out"], 0)
    else:
        st["out"].copy_(_turn(st["x"], st["pos"], c))
    return st["out"]


def _values(codes, code):
    return codes.view(torch.int8 if code == "i8" else torch.float8_e4m3fn).float()


def _read(st, c, x, slots):
    """Values of slots [B, n] of every head: float32 [B, H, n, d]"""
    at = st["table"].gather(1, slots // c["page"]).long()
    rows = st[x][at, :, slots % c["page"]]                                          # [B, n, H, d]
    return (_values(rows, c["code"]) * st[x + "_scale"][at][..., None]).transpose(1, 2)


def _read_lists(st, c):
    B, H = c["B"], c["H"]
    idx = st["sel_idx"].view(B, H, -1).long()
    at = st["table"].long()[:, None].expand(-1, H, -1).gather(2, idx // c["page"])
    head = torch.arange(H, device="cuda")[:, None]
    there = torch.arange(idx.shape[2], device="cuda") < st["sel_cnt"][:, None]
    for x in "KV":
        rows = _values(st[x][at, head, idx % c["page"]], c["code"]) * st[x + "_scale"][at, head][..., None]
        to = st[x + "_sel"]
        to.copy_(torch.where(there[..., None], rows.reshape(to.shape), to.float()))


def _run_append(st, c):
    B, H, T, page = c["B"], c["H"], c["n_rows"], c["page"]
    if own:
        stride = (c["group"] + 2) * H * c["d"] if c["fused"] else 0
        q, k, v = (st[x].data_ptr() if c["fused"] else st[x] for x in "qkv")
        _ctx.ig_append_pages(st["desc"], st["pages"], st["rotary"], c["group"], T, q, k, v, stride, st["n_append"], st["kv_len"],
                             st["pos"], st["q_out"])
        _ctx.ig_gather_pages(st["read"], st["pages"], st["sel_idx"], st["sel_idx"].shape[1], st["sel_cnt"], st["K_sel"], st["V_sel"])
        return dict(q=st["q_out"], K=st["K_sel"], V=st["V_sel"])
    j = torch.arange(T, device="cuda")
    valid = j < st["n_append"][:, None]                                             # [B, T]
    pos = (st["pos"][:, None] + j).view(-1)
    q = _turn(st["q"].reshape(B * T, -1, c["d"]), pos, c).view(st["q_out"].shape)
    st["q_out"].copy_(torch.where(valid[..., None, None], q, st["q_out"].float()))
    k = _turn(st["k"].reshape(B * T, H, c["d"]), pos, c).view(B, T, H, c["d"])
    slot = st["kv_len"][:, None] + j
    b, j = valid.nonzero(as_tuple=True)
    at, most = slot[b, j].long(), _MOST[c["code"]]
    first = st["kv_len"].long() // page                                             # a page that holds rows already, if ..
    held = (st["kv_len"] % page > 0) & (st["n_append"] > 0)
    hb = held.nonzero(as_tuple=True)[0]
    hp = st["table"][hb, first[hb]].long()
    p = st["table"][b, at // page].long()
    for x, rows in (("K", k[b, j]), ("V", st["v"][b, j].float())):
        # the smallest power of two that brings a page's rows within the codes
        top = torch.zeros_like(st["K_scale"]).index_reduce_(0, p, rows.abs().amax(-1), "amax").double() / most
        m, e = torch.frexp(top)
        need = torch.ldexp(torch.ones_like(top), torch.where(m == 0.5, e - 1, e)).clamp_(min=_LEAST).float()
        new, old = st[x + "_scale"].clone(), st[x + "_scale"]
        new[p] = need[p]
        new[hp] = torch.maximum(old[hp], need[hp])
        # the held rows of such a page in its new scale
        before = _values(st[x][hp], c["code"]) * (old[hp] / new[hp])[..., None, None]
        st[x][hp] = torch.where((torch.arange(page, device="cuda") < (st["kv_len"][hb] % page)[:, None])[:, None, :, None],
                                _rounded(before, c["code"]), st[x][hp])
        st[x][p, :, at % page] = _rounded(rows / new[p][..., None], c["code"])
        st[x + "_scale"].copy_(new)
    _read_lists(st, c)
    return dict(q=st["q_out"], K=st["K_sel"], V=st["V_sel"])


def _rounded(x, code):
    """The nearest codes, ties to the even one, as bytes"""
    return x.round().to(torch.int8).view(torch.uint8) if code == "i8" else x.to(torch.float8_e4m3fn).view(torch.uint8)


def _run_gather(st, c):
    if own:
        _ctx.ig_gather_pages(st["read"], st["pages"], st["sel_idx"], st["sel_idx"].shape[1], st["sel_cnt"], st["K_sel"], st["V_sel"])
    else:
        _read_lists(st, c)
    return dict(K=st["K_sel"], V=st["V_sel"])


def _run_attention(st, c):
    B, H, G, T, N, d = c["B"], c["H"], c["group"], c["n_q"], c["N"], c["d"]
    if own:
        _ctx.ig_page_attention(st["desc"], st["pages"], G, T, st["q"], st["q_len"], st["kv_len"], st["out"])
        return st["out"]
    slots = torch.arange(N, device="cuda")
    K, V = (_read(st, c, x, slots.expand(B, -1)).contiguous() for x in "KV")
    i = torch.arange(T, device="cuda")
    last = st["kv_len"][:, None] - st["q_len"][:, None] + i                         # [B, T]
    valid = i < st["q_len"][:, None]
    seen = (slots <= last[:, :, None]) & valid[:, :, None]
    seen = seen[:, None].repeat_interleave(G, 2)                                    # [B, 1, T*G, N]
    q = st["q"].float().view(B, T, H, G, d).permute(0, 2, 1, 3, 4).reshape(B, H, T * G, d)
    logits = (q @ K.transpose(2, 3).contiguous()).mul_(st["scale"]).masked_fill_(~seen, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = logits.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p @ V) / torch.where(total == 0, torch.ones_like(total), total)
    out = out.view(B, H, T, G, d).permute(0, 2, 1, 3, 4).reshape(B, T, H * G, d)
    st["out"].copy_(torch.where(valid[:, :, None, None], out, st["out"].float()))
    return st["out"]


def _pairs(case):
    """Pairs of a query token and a slot it sees, over the batch (one head)."""
    total = 0
    for n, m in zip(*_lengths(case)):
        first = n - m + 1                          # slots the first query sees, may be below 1
        lo = max(first, 1)
        total += (lo + n) * (n - lo + 1) // 2 if n >= lo else 0
    return total


def work(case):
    d, B = case["d"], case["B"]
    row = d * (4 if case["dtype"] == "f32" else 2)
    if case["op"] == "rotate":
        n = B * case["n"]
        return {"bytes": n * (2 * case["heads"] * row + 4) + case["dims"] * 4, "flops": n * case["heads"] * case["dims"] * 3}
    H, page = case["H"], case["page"]
    kv, rows = _lengths(case)
    if case["op"] == "attention":
        Hq = H * case["group"]
        scales = sum((n + page - 1) // page for n in kv) * (H * 8 + 4)
        return {"bytes": sum(kv) * H * 2 * d + scales + sum(rows) * Hq * 2 * row, "flops": 4 * d * Hq * _pairs(case)}
    if case["op"] == "append":
        # queries in and out, keys and values in and as codes out; and what is read back of the pages: codes and values
        Hq, n = H * case["group"], sum(rows)
        back = sum(m + k % page for k, m in zip(kv, rows))
        scales = sum((k % page + m + page - 1) // page for k, m in zip(kv, rows)) * H * 8
        return {"bytes": n * (2 * Hq * row + 2 * H * row + 2 * H * d) + back * H * 2 * (d + 2 * d) + 2 * scales,
                "flops": n * (Hq + H) * case["dims"] * 3 + n * 2 * H * d * 2}
    # (three quarters to all of the rows of every list)
    n = B * H * case["rows"] * 7 / 8
    return {"bytes": int(n * (2 * d + 2 * row + 4)), "flops": int(n * 2 * d)}


def exact(case, seed):
    """What `run` returns, from the definitions: sequence by sequence, in 64 bits."""
    st = _inputs(case, seed)
    d, B = case["d"], case["B"]
    if case["op"] == "rotate":
        return _turn_exact(st["x"].double(), st["pos"], case)
    H, page, code = case["H"], case["page"], case["code"]
    kv, rows = _lengths(case)
    table = st["table"].tolist()
    kind = torch.int8 if code == "i8" else torch.float8_e4m3fn

    def sequence(x, b, n):
        """All heads' values of the first n slots: [H, n, d]"""
        pages = table[b][:(n + page - 1) // page]
        v = st[x][pages].view(kind).double() * st[x + "_scale"][pages].double()[:, :, None, None]
        return v.transpose(0, 1).reshape(H, -1, d)[:, :n]

    if case["op"] == "attention":
        G, out = case["group"], st["out"].double()
        for b in range(B):
            n, m = kv[b], rows[b]
            K, V = sequence("K", b, n), sequence("V", b, n)
            sees = torch.ones((m, n), dtype=torch.bool, device="cuda").tril(n - m)
            for h in range(H * G):
                t = torch.where(sees, st["q"][b, :m, h].double() @ K[h // G].T * (st["scale"] / math.log(2.0)), -math.inf)
                lse = torch.logsumexp(t * math.log(2.0), 1, keepdim=True) / math.log(2.0)
                out[b, :m, h] = torch.where(sees, torch.exp2(t - lse), 0.0) @ V[h // G]
        return out
    if case["op"] == "gather":
        read = {}
        for x in "KV":
            to = st[x + "_sel"].double()
            for b in range(B):
                values = sequence(x, b, case["N"])
                for h in range(H):
                    i = b * H + h
                    n = int(st["sel_cnt"][i])
                    to[i, :n] = values[h, st["sel_idx"][i, :n].long()]
            read[x] = to
        return read
    q = st["q_out"].double()
    to = {x: st[x + "_sel"].double() for x in "KV"}
    for b in range(B):
        n, m = kv[b], rows[b]
        pos = int(st["pos"][b]) + torch.arange(m, device="cuda")
        q[b, :m] = _turn_exact(st["q"][b, :m].double(), pos, case)
        new = {"K": _turn_exact(st["k"][b, :m].double(), pos, case), "V": st["v"][b, :m].double()}
        for x in "KV":
            start = n - n % page
            held = sequence(x, b, n)[:, start:]
            span = torch.cat([held, new[x].transpose(0, 1)], 1)                      # [H, slots of the touched pages, d]
            for p in range((span.shape[1] + page - 1) // page):
                block = span[:, p * page:(p + 1) * page]
                fresh = block[:, n % page:] if p == 0 else block
                need = fresh.abs().amax((1, 2)) / _MOST[code]
                step = torch.exp2(torch.ceil(torch.log2(need.clamp(min=_LEAST))))
                if p == 0 and n % page:
                    step = torch.maximum(step, st[x + "_scale"][table[b][n // page]].double())
                v = block / step[:, None, None]
                if code == "i8":
                    v = v.round()
                else:       # three bits behind the leading one, down to 2^-9
                    unit = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
                    v = (v / unit).round() * unit
                at = p * page
                to[x].view(B, H, -1, d)[b, :, at:at + block.shape[1]] = v * step[:, None, None]
    return dict(q=q, K=to["K"], V=to["V"])


def _turn_exact(x, pos, case):
    """x [n, heads, d] in 64 bits: every pair as a complex number times magnitude e^(i angle)"""
    f, magnitude = _frequencies(case)
    angle = pos.double()[:, None] * f.to(x.device) * (-1 if case.get("inverse") else 1)
    turn = torch.polar(torch.full_like(angle, magnitude), angle)[:, None]
    dims, out = case["dims"], x.clone()
    first = slice(0, dims, 2) if case["interleaved"] else slice(0, dims // 2)
    second = slice(1, dims, 2) if case["interleaved"] else slice(dims // 2, dims)
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _inputs(case, seed):
    """The inputs alone, without the library's descriptors."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was
