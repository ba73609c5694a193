"""What one decoding step over a paged key-value cache is judged by: the four operators that such a step adds to the
PWL forward pass, from one token of one request to a full batch.

  plan    block tables and slot maps from request lengths: Context.kv_plan
  rope    norms of queries and keys for each head (PWL rsqrt), the position rotation and the write to the cache in one
          pass: Context.qk_norm_rope_pwl
  attend  attention of one new token per request over the paged cache with PWL softmax: Context.attention_pwl_paged
  w4      few tokens times 4-bit weights with group scales, PWL epilogue: Context.linear_pwl_w4

Where `own` is false the same results come from elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False

TORCH_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # the next token of every request of a serving batch: lengths grow by one, some requests end, some join
        plan("plan_decode_b256", B=256, page=16, width=128, new=1),
        # a step that takes in whole prompts beside running requests
        plan("plan_prompts_b1024", B=1024, page=64, width=256, new=512),
        # one token of one request: launch latency
        rope("rope_one_token_f32", "f32", T=1, heads=12, kv_heads=12, d=64, rot=64, page=16),
        # the tokens of a decoding batch, padded to a round number as a captured graph wants it
        rope("rope_decode_f16", "f16", T=192, heads=32, kv_heads=8, d=128, rot=128, page=64),
        # prompts: bound by the bytes of the projection
        rope("rope_prompts_bf16", "bf16", T=16383, heads=32, kv_heads=8, d=128, rot=64, page=16, pairs=True),
        # one request with the heads of the BERT-base shape, a few hundred tokens long
        attend("attend_one_request_bf16", "bf16", B=1, L=500, heads=12, kv_heads=12, d=64, page=16),
        # the fp32 evaluation of a small batch
        attend("attend_batch_f32", "f32", B=6, L=1333, heads=16, kv_heads=4, d=64, page=32),
        # one request with a book in its cache: few rows, a very long axis
        attend("attend_long_f16", "f16", B=1, L=131071, heads=32, kv_heads=8, d=128, page=64),
        # a full serving batch of requests of very different lengths
        attend("attend_full_batch_bf16", "bf16", B=48, L=8192, heads=32, kv_heads=8, d=128, page=16),
        # one token through the first FFN matrix of the BERT-large shape, GELU table in the epilogue
        w4("w4_one_token_bf16", "bf16", M=1, N=4096, K=1024, group=64, slot=True),
        # a handful of requests through a square projection with bias and residual
        w4("w4_few_tokens_f16", "f16", M=7, N=4100, K=4096, group=128, residual=True),
        # a decoding batch through a wide matrix: bound by the weights' bytes
        w4("w4_batch_bf16", "bf16", M=32, N=16384, K=8192, group=128),
    ]


def draw(rng):
    kind = rng.choice(["plan", "rope", "rope", "attend", "attend", "attend", "w4", "w4"])
    if kind == "plan":
        page = rng.choice([8, 16, 32, 64, 100])
        B = log_int(rng, 1, 1024)
        return plan(None, B, page, width=rng.choice([64, 100, 256]), new=rng.choice([1, 1, log_int(rng, 2, 512)]), mix=rng.randrange(1 << 16))
    if kind == "rope":
        d = rng.choice([64, 64, 96, 128, 128, 256])
        kv_heads = rng.choice([1, 2, 4, 8])
        heads = kv_heads * rng.choice([1, 2, 4, 7, 8])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        top = (1 << 28) // ((heads + 2 * kv_heads) * d * BYTES[dtype])
        return rope(None, dtype, log_int(rng, 1, min(16383, top)), heads, kv_heads, d, rot=rng.choice([d, d, d // 2]), page=rng.choice([16, 64, 33]),
                    pairs=rng.random() < 0.3, norm=rng.random() < 0.8, mix=rng.randrange(1 << 16))
    if kind == "attend":
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        d = rng.choice([64, 64, 128, 128, 96])
        kv_heads = rng.choice([1, 2, 4, 8, 12])
        heads = kv_heads * rng.choice([1, 1, 4, 5, 8, 16])
        # K and V take no more than a third of the largest listed case's
        top = (1 << 28) // (kv_heads * d * 2 * BYTES[dtype])
        L = log_int(rng, 1, min(131072, top))
        top //= L
        return attend(None, dtype, log_int(rng, 1, min(128, top)), L, heads, kv_heads, d, page=rng.choice([8, 16, 32, 64, 128, 24]), mix=rng.randrange(1 << 16))
    K = 128 * log_int(rng, 2, 64)
    group = rng.choice([32, 64, 128, 128])
    if rng.random() < 0.3:
        K -= 128 - group
    N = log_int(rng, 256, 16384)
    return w4(None, rng.choice(["bf16", "bf16", "f16", "f32"]), log_int(rng, 1, 32), N if rng.random() < 0.3 else (N + 7) // 8 * 8, K, group,
              slot=rng.random() < 0.5, residual=rng.random() < 0.5)


def log_int(rng, lo, hi):
    """A whole number from lo to hi, its logarithm uniform."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def named(name, case):
    return case if name is None else dict(case, name=name)


def plan(name, B, page, width, new, mix=0):
    return named(name, {"kind": "plan", "B": B, "page": page, "width": width, "new": new, "mix": mix})


def rope(name, dtype, T, heads, kv_heads, d, rot, page, pairs=False, norm=True, mix=0):
    return named(name, {"kind": "rope", "dtype": dtype, "T": T, "heads": heads, "kv_heads": kv_heads, "d": d, "rot": rot, "page": page,
                        "pairs": pairs, "norm": norm, "mix": mix})


def attend(name, dtype, B, L, heads, kv_heads, d, page, mix=0):
    return named(name, {"kind": "attend", "dtype": dtype, "B": B, "L": L, "heads": heads, "kv_heads": kv_heads, "d": d, "page": page, "mix": mix})


def w4(name, dtype, M, N, K, group, slot=False, residual=False):
    return named(name, {"kind": "w4", "dtype": dtype, "M": M, "N": N, "K": K, "group": group, "slot": slot, "residual": residual})


# ---------------------------------------------------------------- lengths, tables


def lengths_of(case):
    """Attention: tokens in each request's cache.  One request has the longest, the others anything up to it; in a larger
    batch one place is empty."""
    rng = random.Random(case["mix"] * 131 + case["L"] * 7 + case["B"])
    lens = [case["L"]] + [rng.randint(1, case["L"]) for _ in range(case["B"] - 1)]
    if case["B"] > 4:
        lens[-2] = 0
    return lens


def steps_of(case):
    """Plan: tokens that the requests have and tokens that the step adds (-1: the request is over).  Some places are empty."""
    rng = random.Random(case["mix"] * 131 + case["B"])
    have, new = [], []
    room = case["width"] * case["page"]
    for _ in range(case["B"]):
        n = case["new"] if case["new"] == 1 or rng.random() < 0.1 else rng.randint(0, case["new"])
        h = 0 if rng.random() < 0.1 else rng.randint(0, max(0, room - n))
        have.append(h)
        new.append(-1 if rng.random() < 0.08 else min(n, room - h))
    return have, new


def secant_table(f, n, lo, hi):
    """n segments of equal width: (k, b) of the line through each segment's end points, rounded to 32 bits, and the index's
    factor and offset."""
    x = lo + (hi - lo) / n * torch.arange(n + 1, dtype=torch.float64)
    y = f(x)
    k = (y[1:] - y[:-1]) / (x[1:] - x[:-1])
    b = y[:-1] - k * x[:-1]
    return {"k": k.float(), "b": b.float(), "n": n, "lo": lo, "hi": hi}


def on_device(t):
    return dict(t, k=t["k"].cuda(), b=t["b"].cuda())


def pwl(t, x):
    """The table at x, inputs outside its range on the end segments' lines."""
    scale = t["n"] / (t["hi"] - t["lo"])
    s = torch.clamp(torch.floor(x * scale - t["lo"] * scale), 0, t["n"] - 1).long()
    return t["k"].to(x.dtype)[s] * x + t["b"].to(x.dtype)[s]


def gelu(x):
    return 0.5 * x * (1.0 + torch.erf(x / math.sqrt(2.0)))


# ---------------------------------------------------------------- preparation


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"plan": prepare_plan, "rope": prepare_rope, "attend": prepare_attend, "w4": prepare_w4}[case["kind"]](case, gen)
    s["case"] = case
    s["tables"] = {name: on_device(t) for name, t in s["host_tables"].items()}
    if own:
        import paper_2305_14405_b200 as nm
        ctx = s["ctx"] = nm.Context(torch.cuda.current_device())
        for name, t in s["host_tables"].items():
            ctx.pwl_table_load(getattr(nm, "SLOT_" + name.upper()), t["n"], t["lo"], t["hi"], t["k"].tolist(), t["b"].tolist())
        {"plan": own_plan, "rope": own_rope, "attend": own_attend, "w4": own_w4}[case["kind"]](nm, ctx, case, s)
    return s


def normal(gen, shape, std=1.0, mean=0.0):
    return torch.randn(shape, generator=gen, device=gen.device) * std + mean


def whole(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def pages_of(tokens, page):
    return -(-tokens // page)


def prepare_plan(case, gen):
    B, page, width = case["B"], case["page"], case["width"]
    have, new = steps_of(case)
    used = [pages_of(h, page) for h in have]
    spare = sum(pages_of(h + max(n, 0), page) - u for h, n, u in zip(have, new, used)) + 5
    pages = sum(used) + spare
    order = torch.randperm(pages, generator=gen, device=gen.device).to(torch.int32)
    tables = torch.full((B, width), -1, dtype=torch.int32, device=gen.device)
    held = torch.arange(width, device=gen.device)[None, :] < whole(used)[:, None]
    tables[held] = order[:sum(used)]
    free = torch.full((pages,), -1, dtype=torch.int32, device=gen.device)
    free[:spare] = order[sum(used):]
    tokens = sum(max(n, 0) for n in new)
    top = max(8, -(-tokens // 8) * 8)   # the arrays of a captured step are of a round size
    return {"host_tables": {}, "lengths": whole(have), "new": whole(new), "block_tables": tables, "free": free, "free_count": whole([spare]),
            "top": top}


def own_plan(nm, ctx, case, s):
    empty = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")  # noqa: E731
    s["out"] = {"lengths": empty(case["B"]), "free_count": empty(1), "token_start": empty(case["B"] + 1), "slots": empty(s["top"]),
                "positions": empty(s["top"]), "block_tables": s["block_tables"], "free": s["free"]}
    o = s["out"]
    s["desc"] = ctx.kv_plan_desc(s["lengths"], s["new"], s["block_tables"], s["free"], s["free_count"], case["page"], o["lengths"],
                                 o["free_count"], o["token_start"], o["slots"], o["positions"])


def prepare_rope(case, gen):
    T, hq, hk, d, page, td = case["T"], case["heads"], case["kv_heads"], case["d"], case["page"], TORCH_DTYPE[case["dtype"]]
    longest = 32768
    qkv = normal(gen, (T, (hq + 2 * hk) * d)).to(td)
    pages = pages_of(T, page) + 2
    slots = torch.randperm(pages * page, generator=gen, device=gen.device)[:T].to(torch.int32)
    if T > 8:
        slots[T - T % 5:] = -1   # rows behind the last token
    cache = lambda: normal(gen, (pages, page, hk, d)).to(td)  # noqa: E731
    rate = 10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device=gen.device) / case["rot"])
    angle = torch.arange(longest, dtype=torch.float64, device=gen.device)[:, None] * rate
    return {"host_tables": {"rsqrt": secant_table(torch.rsqrt, 64, 0.25, 4.0)}, "qkv": qkv, "k_cache": cache(), "v_cache": cache(),
            "slots": slots, "positions": torch.randint(0, longest, (T,), generator=gen, device=gen.device, dtype=torch.int32),
            "cos_sin": torch.cat([torch.cos(angle), torch.sin(angle)], dim=1).float(),
            "gamma_q": normal(gen, (d,), 0.1, 1.0) if case["norm"] else None, "gamma_k": normal(gen, (d,), 0.1, 1.0) if case["norm"] else None,
            "q_out": torch.zeros((T, hq * d), dtype=td, device=gen.device)}


def own_rope(nm, ctx, case, s):
    s["desc"] = ctx.qk_rope_desc(s["qkv"], case["heads"], case["kv_heads"], case["d"], s["q_out"], positions=s["positions"], cos_sin=s["cos_sin"],
                                 gamma_q=s["gamma_q"], gamma_k=s["gamma_k"], eps=1e-6, pairs=case["pairs"], k_cache=s["k_cache"],
                                 v_cache=s["v_cache"], slots=s["slots"])


def prepare_attend(case, gen):
    B, hk, d, page, td = case["B"], case["kv_heads"], case["d"], case["page"], TORCH_DTYPE[case["dtype"]]
    lens = lengths_of(case)
    used = [pages_of(n, page) for n in lens]
    pages = sum(used) + 3
    order = torch.randperm(pages, generator=gen, device=gen.device).to(torch.int32)
    width = pages_of(case["L"], page)
    tables = torch.zeros((B, width), dtype=torch.int32, device=gen.device)
    held = torch.arange(width, device=gen.device)[None, :] < whole(used)[:, None]
    tables[held] = order[:sum(used)]

    def cache():
        c = torch.empty((pages, page, hk, d), dtype=td, device=gen.device)
        step = max(1, (1 << 26) // (page * hk * d))
        for i in range(0, pages, step):
            c[i:i + step] = normal(gen, (min(step, pages - i), page, hk, d)).to(td)
        return c

    L = case["L"]
    return {"host_tables": {"exp": secant_table(torch.exp, 256, -16.0, 0.0), "recip": secant_table(lambda x: 1.0 / x, 256, max(0.25, L / 256.0), L + 1.0)},
            "q": normal(gen, (B, case["heads"], d)).to(td), "k_cache": cache(), "v_cache": cache(), "block_tables": tables, "lengths": whole(lens)}


def own_attend(nm, ctx, case, s):
    s["out"] = torch.empty_like(s["q"])
    s["desc"] = ctx.attn_paged_desc(s["q"], s["k_cache"], s["v_cache"], s["block_tables"], s["lengths"], s["out"], max_len=case["L"])
    s["workspace"] = torch.empty(ctx.attention_paged_workspace_bytes(s["desc"]), dtype=torch.uint8, device="cuda")


def prepare_w4(case, gen):
    M, N, K, td = case["M"], case["N"], case["K"], TORCH_DTYPE[case["dtype"]]
    wide = -(-N // 8) * 8   # rows of whole 16-byte pieces
    return {"host_tables": {"gelu": secant_table(gelu, 64, -4.0, 4.0)}, "a": normal(gen, (M, K)).to(td),
            "codes": torch.randint(0, 256, (N, K // 2), generator=gen, device=gen.device, dtype=torch.uint8),
            "scales": (normal(gen, (N, K // case["group"]), 0.1, 1.0) * 0.2 / math.sqrt(K)).to(td), "bias": normal(gen, (N,), 0.02),
            "residual": normal(gen, (M, wide)).to(td)[:, :N] if case["residual"] else None}


def own_w4(nm, ctx, case, s):
    wide = -(-case["N"] // 8) * 8
    s["out"] = torch.empty((case["M"], wide), dtype=s["a"].dtype, device="cuda")[:, :case["N"]]
    s["desc"] = ctx.linear_w4_desc(s["a"], s["codes"], s["scales"], s["out"], bias=s["bias"], residual=s["residual"],
                                   slot=nm.SLOT_GELU if case["slot"] else nm.SLOT_NONE)


# ---------------------------------------------------------------- one pass


def run(s):
    kind = s["case"]["kind"]
    if own:
        ctx, desc = s["ctx"], s["desc"]
        if kind == "plan":
            ctx.kv_plan(desc)
            return s["out"]
        if kind == "rope":
            ctx.qk_norm_rope_pwl(desc)
            return s["q_out"], s["k_cache"], s["v_cache"]
        if kind == "attend":
            ctx.attention_pwl_paged(desc, s["workspace"])
            return s["out"]
        ctx.linear_pwl_w4(desc)
        return s["out"]
    return {"plan": plain_plan, "rope": plain_rope, "attend": plain_attend, "w4": plain_w4}[kind](s, s["case"])


def plain_plan(s, case):
    B, page, width, top = case["B"], case["page"], case["width"], s["top"]
    lengths, new = s["lengths"].long(), s["new"].long()
    over = new < 0
    held, add = -(-lengths // page), torch.clamp(new, min=0)
    after = torch.where(over, 0, lengths + add)
    released = torch.where(over, held, 0)
    wanted = torch.where(over, 0, -(-after // page) - held)
    column = torch.arange(width, device=lengths.device)[None, :]
    tables, free = s["block_tables"].clone(), s["free"].clone()
    # released pages go on the stack in the requests' order
    count = s["free_count"].long()
    put = (column < released[:, None])
    at = count + torch.cumsum(released, 0)[:, None] - released[:, None] + column
    free[at[put]] = tables[put]
    stack = count + released.sum()
    # the k-th new page is the k-th from the stack's top
    take = (column >= held[:, None]) & (column < (held + wanted)[:, None])
    nth = torch.cumsum(wanted, 0)[:, None] - wanted[:, None] + column - held[:, None]
    tables[take] = free[(stack - 1 - nth)[take]]
    start = torch.cat([torch.zeros_like(lengths[:1]), torch.cumsum(torch.where(over, 0, add), 0)])
    token = torch.arange(top, device=lengths.device)
    request = torch.clamp(torch.searchsorted(start, token, right=True) - 1, max=B - 1)
    live = token < start[-1]
    position = torch.where(live, lengths[request] + token - start[request], 0)
    slot = torch.where(live, tables[request, torch.clamp(position // page, max=width - 1)].long() * page + position % page, -1)
    whole32 = lambda x: x.to(torch.int32)  # noqa: E731
    return {"lengths": whole32(after), "free_count": whole32(stack - wanted.sum()), "token_start": whole32(start), "slots": whole32(slot),
            "positions": whole32(position), "block_tables": tables, "free": free}


def turned(x, cos, sin, rot, pairs):
    """The first `rot` channels of every head rotated, two neighbours at a time or the first half with the second."""
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if pairs else (r[..., :rot // 2], r[..., rot // 2:])
    u, v = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([u, v], dim=-1).flatten(-2) if pairs else torch.cat([u, v], dim=-1)
    return torch.cat([y, x[..., rot:]], dim=-1)


def plain_rope(s, case):
    T, hq, hk, d, td = case["T"], case["heads"], case["kv_heads"], case["d"], s["qkv"].dtype
    x = s["qkv"].float().view(T, hq + 2 * hk, d)
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    if case["norm"]:
        q = q * pwl(s["tables"]["rsqrt"], (q * q).mean(-1, keepdim=True) + 1e-6) * s["gamma_q"]
        k = k * pwl(s["tables"]["rsqrt"], (k * k).mean(-1, keepdim=True) + 1e-6) * s["gamma_k"]
    row = s["cos_sin"][s["positions"].long()]
    cos, sin = row[:, None, :case["rot"] // 2], row[:, None, case["rot"] // 2:]
    q, k = turned(q, cos, sin, case["rot"], case["pairs"]), turned(k, cos, sin, case["rot"], case["pairs"])
    at = torch.nonzero(s["slots"] >= 0)[:, 0]
    slot = s["slots"][at].long()
    s["q_out"][at] = q[at].reshape(-1, hq * d).to(td)
    s["k_cache"].view(-1, hk, d)[slot] = k[at].to(td)
    s["v_cache"].view(-1, hk, d)[slot] = v[at].to(td)
    return s["q_out"], s["k_cache"], s["v_cache"]


def plain_attend(s, case):
    B, L, hq, hk, d = case["B"], case["L"], case["heads"], case["kv_heads"], case["d"]
    pages = s["block_tables"].long()
    gather = lambda c: c[pages].view(B, -1, hk, d)[:, :L].permute(0, 2, 1, 3).float()  # noqa: E731
    live = torch.arange(L, device=pages.device)[None, None, None, :] < s["lengths"][:, None, None, None]
    q = s["q"].float().view(B, hk, hq // hk, d)
    x = torch.matmul(q, gather(s["k_cache"]).transpose(2, 3)) * d ** -0.5
    m = torch.where(live, x, -math.inf).amax(-1, keepdim=True)
    e = torch.where(live, pwl(s["tables"]["exp"], torch.where(live, x - m, 0.0)), 0.0)
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e, gather(s["v_cache"])) * pwl(s["tables"]["recip"], total)
    o = torch.where(s["lengths"][:, None, None, None] > 0, o, 0.0)
    return o.reshape(B, hq, d).to(s["q"].dtype)


def values_of(codes):
    """The 4-bit codes of each row, the low half of a byte first, as whole numbers from -8 to 7."""
    return torch.stack([codes & 15, codes >> 4], dim=-1).flatten(1).to(torch.int8) - 8


def plain_w4(s, case):
    N, K, group = case["N"], case["K"], case["group"]
    w = (values_of(s["codes"]).float().view(N, K // group, group) * s["scales"].float()[:, :, None]).view(N, K)
    y = torch.matmul(s["a"].float(), w.t()) + s["bias"]
    if case["slot"]:
        y = pwl(s["tables"]["gelu"], y)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["a"].dtype)


# ---------------------------------------------------------------- the same in 64 bits


def line_at(t, x):
    """The table at x in 64 bits: the segment by search among the borders."""
    border = torch.linspace(t["lo"], t["hi"], t["n"] + 1, dtype=torch.float64, device=x.device)[1:-1]
    s = torch.searchsorted(border, x.contiguous(), right=True)
    return torch.addcmul(t["b"].double()[s], t["k"].double()[s], x)


def exact(case, seed):
    if case["kind"] == "plan":
        return None
    s = prepare(case, seed)
    t = s["tables"]
    if case["kind"] == "rope":
        T, hq, hk, d, half = case["T"], case["heads"], case["kv_heads"], case["d"], case["rot"] // 2
        q_out, caches = s["q_out"].double(), [s["k_cache"].double(), s["v_cache"].double()]
        rows = (s["slots"] >= 0).nonzero().flatten()
        rows_at = s["slots"][rows].long()
        at = s["cos_sin"].double()[s["positions"][rows].long()]
        x = s["qkv"].double().view(T, -1, d)[rows]
        # channel pairs that turn together, as complex numbers
        first = torch.arange(half, device=x.device) * (2 if case["pairs"] else 1)
        second = first + (1 if case["pairs"] else half)
        angle = torch.complex(at[:, :half], at[:, half:])[:, None, :]
        for part, gamma in ((slice(0, hq), s["gamma_q"]), (slice(hq, hq + hk), s["gamma_k"])):
            y = x[:, part]
            if case["norm"]:
                y = y * line_at(t["rsqrt"], y.square().sum(-1, keepdim=True) / d + 1e-6) * gamma.double()
            z = torch.complex(y[..., first], y[..., second]) * angle
            x[:, part] = y
            x[:, part, :].index_copy_(2, first, z.real)
            x[:, part, :].index_copy_(2, second, z.imag)
        q_out[rows] = x[:, :hq].flatten(1)
        caches[0].view(-1, hk, d)[rows_at] = x[:, hq:hq + hk]
        caches[1].view(-1, hk, d)[rows_at] = x[:, hq + hk:]
        return q_out, caches[0], caches[1]
    if case["kind"] == "attend":
        hk, d, g = case["kv_heads"], case["d"], case["heads"] // case["kv_heads"]
        out = torch.zeros((case["B"], case["heads"], d), dtype=torch.float64, device="cuda")
        for i, n in enumerate(lengths_of(case)):
            if n == 0:
                continue
            token = torch.arange(n, device="cuda")
            page, place = s["block_tables"][i].long()[token // case["page"]], token % case["page"]
            for h in range(hk):
                k, v = s["k_cache"][page, place, h].double(), s["v_cache"][page, place, h].double()
                x = (s["q"][i, h * g:(h + 1) * g].double() @ k.t()) / math.sqrt(d)
                e = line_at(t["exp"], x - x.max(1, keepdim=True).values)
                out[i, h * g:(h + 1) * g] = (e @ v) * line_at(t["recip"], e.sum(1, keepdim=True))
        return out
    a, codes, group = s["a"].double(), s["codes"], case["group"]
    y = torch.empty((case["M"], case["N"]), dtype=torch.float64, device="cuda")
    for i in range(0, case["N"], 2048):
        c = codes[i:i + 2048].to(torch.int64)
        w = torch.empty((c.shape[0], case["K"]), dtype=torch.float64, device="cuda")
        w[:, 0::2], w[:, 1::2] = (c % 16 - 8).double(), (c // 16 - 8).double()
        y[:, i:i + 2048] = a @ (w * s["scales"][i:i + 2048].double().repeat_interleave(group, dim=1)).t()
    y += s["bias"].double()
    if case["slot"]:
        y = line_at(t["gelu"], y)
    return y if s["residual"] is None else y + s["residual"].double()


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    if case["kind"] == "plan":
        have, new = steps_of(case)
        page = case["page"]
        tokens = sum(max(n, 0) for n in new)
        moved = sum(pages_of(h, page) if n < 0 else pages_of(h + n, page) - pages_of(h, page) for h, n in zip(have, new))
        # lengths and steps in, lengths and starts out, every moved page read and written, the old page of every token's request, slots and positions
        return {"bytes": 4 * (4 * case["B"] + 2 * moved + case["B"] + 2 * tokens), "flops": 2 * tokens + 8 * case["B"]}
    es = BYTES[case["dtype"]]
    if case["kind"] == "rope":
        T, d, hq, hk = case["T"], case["d"], case["heads"], case["kv_heads"]
        return {"bytes": T * (2 * (hq + 2 * hk) * d * es + 4 * case["rot"] + 8), "flops": T * (hq + hk) * d * 8}
    if case["kind"] == "attend":
        tokens, d = sum(lengths_of(case)), case["d"]
        return {"bytes": tokens * case["kv_heads"] * d * 2 * es + 4 * (tokens // case["page"]) + 2 * case["B"] * case["heads"] * d * es,
                "flops": 4 * tokens * case["heads"] * d}
    M, N, K = case["M"], case["N"], case["K"]
    return {"bytes": N * K // 2 + N * (K // case["group"]) * es + 4 * N + (M * K + M * N * (2 if case["residual"] else 1)) * es, "flops": 2 * M * N * K}
