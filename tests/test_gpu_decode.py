"""GPU parity of the operators of one decoding step over a paged key-value cache, against 64-bit references."""
import numpy as np
import pytest
import torch

import decode_ref as ref
from decode_ref import TYPES, check, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(nm):
    c = nm.Context(0)
    c.tabs = ref.load_tables(c)
    yield c
    c.close()


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def gen_of(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# ---------------------------------------------------------------- plan


class Plan:
    """Arrays of one step, with canaries behind each."""

    def __init__(self, ctx, lengths, new, page, width, free, count, max_tokens, tables=None, in_place=False, pad=3):
        B = len(lengths)
        rng = np.random.default_rng(B * 7 + page)
        self.host_tables = rng.integers(0, 1 << 20, (B, width)).astype(np.int32) if tables is None else tables
        self.wide = torch.full((B, width + pad), -77, dtype=torch.int32, device="cuda")
        self.tables = self.wide[:, :width]
        self.tables.copy_(torch.from_numpy(self.host_tables))
        self.lengths, self.new, self.free, self.count = i32(lengths), i32(new), i32(list(free)), i32([count])
        out = lambda n: torch.full((n + 4,), -77, dtype=torch.int32, device="cuda")  # noqa: E731
        self.raw = {"lengths": out(B), "free_count": out(1), "token_start": out(B + 1), "slots": out(max_tokens), "positions": out(max_tokens)}
        self.out = {k: v[:-4] for k, v in self.raw.items()}
        if in_place:
            self.out["lengths"], self.out["free_count"] = self.lengths, self.count
        o = self.out
        self.ctx, self.page, self.max_tokens = ctx, page, max_tokens
        self.desc = ctx.kv_plan_desc(self.lengths, self.new, self.tables, self.free, self.count, page, o["lengths"], o["free_count"],
                                     o["token_start"], o["slots"], o["positions"])

    def run_and_check(self):
        tables, free = self.tables.cpu().numpy().copy(), self.free.cpu().numpy().copy()
        lengths, new, count = self.lengths.tolist(), self.new.tolist(), int(self.count.item())
        status, want = ref.plan(lengths, new, tables, free, count, self.page, self.max_tokens)
        self.ctx.kv_plan(self.desc)
        assert self.ctx.poll_status() == status
        for k, v in want.items():
            assert self.out[k].tolist() == (v if isinstance(v, list) else [v]), k
        assert np.array_equal(self.tables.cpu().numpy(), tables)
        assert np.array_equal(self.free.cpu().numpy(), free)
        assert (self.wide[:, tables.shape[1]:] == -77).all()
        for k, v in self.raw.items():
            assert (v[-4:] == -77).all(), k
        return status


@pytest.mark.parametrize("B,page,width,new_max", [(1, 16, 4, 1), (3, 1, 40, 9), (31, 16, 8, 1), (256, 16, 128, 1), (1000, 100, 12, 300), (1025, 64, 9, 40),
                                                  (2049, 8, 33, 3), (5, 64, 256, 16000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan(ctx, B, page, width, new_max, in_place):
    rng = np.random.default_rng(B + page)
    room = page * width
    new = np.minimum(rng.integers(0, new_max + 1, B), room)
    lengths = np.array([rng.integers(0, room - n + 1) for n in new])
    lengths[::7] = 0
    if B > 2:
        lengths[-1], new[-1] = room, 0            # a full row that gets nothing
        new[rng.random(B) < 0.2] = -1
        new[1], lengths[1] = -1, room             # the longest release
    need = int(sum(-(-(h + max(n, 0)) // page) for h, n in zip(lengths, new))) + 3
    p = Plan(ctx, lengths.tolist(), new.tolist(), page, width, rng.permutation(need + B * width), need, int(np.maximum(new, 0).sum()) + B % 5, in_place=in_place)
    assert p.run_and_check() == 0
    if in_place:                                  # the next step of the same arrays
        p.new.copy_(i32([int(n) for n in rng.integers(-1, 1, B)]))
        assert p.run_and_check() == 0


def test_plan_takes_released_pages_in_the_same_step(ctx):
    # three free pages, five released ones, seven wanted
    p = Plan(ctx, [80, 3, 16], [-1, 93, 16], 16, 8, [900, 901, 902] + [-1] * 40, 3, 128)
    assert p.run_and_check() == 0
    assert p.out["free_count"].tolist() == [2]


@pytest.mark.parametrize("lengths,new,count,max_tokens,status", [
    ([10, 20], [1, 20], 0, 64, 8),        # a page wanted, none free
    ([10, 20], [1, 45], 9, 64, 2),        # longer than its table row
    ([10, 20], [30, 30], 9, 59, 2),       # more tokens than slots
    ([10, 65], [1, 1], 9, 64, 1),         # a length that its row cannot hold
    ([-1, 6], [1, 1], 9, 64, 1),
    ([10, 20], [1, 1], -1, 64, 1),
    ([10, 20], [1, 1], 41, 64, 1),
    ([10, 20], [-1, -1], 38, 64, 1),      # three pages back on a stack with room for two
    ([10, 2 ** 31 - 1], [2 ** 31 - 1, 2 ** 31 - 1], 9, 64, 1),
    ([10, 20], [2 ** 31 - 1, 2 ** 31 - 1], 9, 64, 2),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan_that_cannot_be_made_changes_nothing(ctx, lengths, new, count, max_tokens, status, in_place):
    p = Plan(ctx, lengths, new, 16, 4, range(40), count, max_tokens, in_place=in_place)
    assert p.run_and_check() == status


def test_plan_gives_no_slot_on_pages_that_have_none(ctx):
    """A negative page, and one whose slots pass 31 bits (2^28 + 3 pages of 16: as 32 bits they would be page 3's)."""
    for bad in (-1, -2 ** 31, 2 ** 27, 2 ** 28 + 3, 2 ** 31 - 1):
        p = Plan(ctx, [0, 16, 30], [2, 3, 4], 16, 4, [7, 8, bad], 3, 12)
        p.tables[2, 1] = bad                      # held: the first two tokens of the third request go there
        ctx.kv_plan(p.desc)
        assert ctx.poll_status() == 1
        assert p.out["slots"].tolist() == [-1, -1, 128, 129, 130, -1, -1, 112, 113, -1, -1, -1]
        assert p.out["positions"].tolist() == [0, 1, 16, 17, 18, 30, 31, 32, 33, 0, 0, 0]
    p = Plan(ctx, [0], [2], 16, 4, [2 ** 27 - 1], 1, 2)
    assert p.run_and_check() == 0
    assert p.out["slots"].tolist() == [2 ** 31 - 16, 2 ** 31 - 15]


def test_plan_of_nothing(ctx):
    p = Plan(ctx, [], [], 16, 4, range(8), 5, 6)
    assert p.run_and_check() == 0
    p = Plan(ctx, [0, 0], [0, 0], 16, 0, [], 0, 0)
    assert p.run_and_check() == 0


# ---------------------------------------------------------------- norm, rotation, cache write


def cache_views(dtype, pages, page, hk, d, layout, fill):
    """K and V as [pages, page, heads, d] views of three layouts."""
    if layout == "token":
        k, v = (torch.full((pages, page, hk, d), fill, dtype=dtype, device="cuda") for _ in range(2))
        return k, v
    if layout == "head":
        k, v = (torch.full((pages, hk, page, d), fill, dtype=dtype, device="cuda").transpose(1, 2) for _ in range(2))
        return k, v
    both = torch.full((pages, 2, page, hk, d + 8), fill, dtype=dtype, device="cuda")   # K and V of a page side by side, rows with a gap
    return both[:, 0, ..., :d], both[:, 1, ..., :d]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,hq,hk,d,rot,pairs,norm,layout", [
    (1, 12, 12, 64, 64, False, "qk", "token"), (1, 1, 1, 8, 8, True, "qk", "token"), (5, 4, 1, 128, 128, False, "qk", "head"),
    (37, 8, 2, 96, 48, False, "q", "both"), (130, 6, 3, 256, 64, True, "k", "both"), (64, 3, 3, 40, 0, False, "qk", "token"),
    (19, 5, 5, 16, 16, False, "", "head"), (700, 32, 8, 128, 64, False, "qk", "token"), (3, 0, 2, 64, 32, True, "qk", "token"),
    (3, 7, 0, 64, 32, False, "qk", "none"), (2000, 2, 1, 72, 16, False, "qk", "token"), (9, 4, 2, 64, 64, False, "qk", "none")])
def test_rope(ctx, dtype, T, hq, hk, d, rot, pairs, norm, layout):
    td, gen, page = TYPES[dtype], gen_of(T + d), 12
    wide = torch.full((T, (hq + 2 * hk) * d + 16), float("nan"), dtype=td, device="cuda")
    qkv = wide[:, :(hq + 2 * hk) * d]
    qkv.copy_(randn(gen, T, (hq + 2 * hk) * d))
    longest = 70000
    positions = torch.randint(0, longest, (T,), generator=gen, device="cuda", dtype=torch.int32)
    angle = torch.rand((longest, max(rot // 2, 1)), generator=gen, device="cuda") * 6.3
    cos_sin = torch.cat([angle.cos(), angle.sin()], 1) if rot else None
    gq = 1 + 0.1 * randn(gen, d) if "q" in norm else None
    gk = 1 + 0.1 * randn(gen, d) if "k" in norm else None
    pages = T // page + 3
    slots = torch.randperm(pages * page, generator=gen, device="cuda")[:T].to(torch.int32)
    slots[T // 2:T // 2 + T // 6] = -1
    kc, vc = cache_views(td, pages, page, hk, d, layout, 7.0) if layout != "none" else (None, None)
    q_wide = torch.full((T, hq * d + 8), 5.0, dtype=td, device="cuda")
    k_wide = torch.full((T, hk * d + 8), 5.0, dtype=td, device="cuda")
    ctx.qk_norm_rope_pwl(ctx.qk_rope_desc(qkv, hq, hk, d, q_wide[:, :hq * d], positions=positions, cos_sin=cos_sin, gamma_q=gq, gamma_k=gk, pairs=pairs,
                                          k_cache=kc, v_cache=vc, slots=slots, k_out=k_wide[:, :hk * d]))
    ctx.check_device_status()
    x, pos, live = f64(qkv).reshape(T, hq + 2 * hk, d), positions.cpu().numpy(), slots.cpu().numpy() >= 0
    cs = f64(cos_sin) if rot else None
    y, dy = x.copy(), np.zeros_like(x)
    for part, g in ((slice(0, hq), gq), (slice(hq, hq + hk), gk)):
        y[:, part], dy[:, part] = ref.rope(x[:, part], pos, cs, None if g is None else f64(g), 1e-6, rot, pairs, ctx.tabs["rsqrt"])
    q, k = (lambda z: z[:, :hq].reshape(T, -1)), (lambda z: z[:, hq:hq + hk].reshape(T, -1))
    check(q_wide[:, :hq * d][live], q(y)[live], q(dy)[live], td, "q")
    check(k_wide[:, :hk * d][live], k(y)[live], k(dy)[live], td, "k")
    for w, n in ((q_wide, hq * d), (k_wide, hk * d)):   # padding rows and the gap behind the rows
        assert (w[:, n:] == 5).all() and (w[:, :n][~torch.from_numpy(live).cuda()] == 5).all()
    if kc is not None:
        at = slots[torch.from_numpy(live).cuda()].long()
        assert torch.equal(kc[at // page, at % page].flatten(1), k_wide[:, :hk * d][torch.from_numpy(live).cuda()])
        assert torch.equal(vc[at // page, at % page].flatten(1), qkv[torch.from_numpy(live).cuda()][:, (hq + hk) * d:])
        rest = torch.ones(pages * page, dtype=torch.bool, device="cuda")
        rest[at] = False
        r = rest.nonzero().flatten()
        assert (kc[r // page, r % page] == 7).all() and (vc[r // page, r % page] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pairs", [False, True])
def test_rope_in_place(ctx, dtype, pairs):
    T, hq, hk, d = 50, 6, 2, 64
    td, gen = TYPES[dtype], gen_of(3)
    qkv = randn(gen, T, (hq + 2 * hk) * d).to(td)
    positions = torch.arange(T, dtype=torch.int32, device="cuda")
    cos_sin = randn(gen, T, d)
    g = 1 + 0.1 * randn(gen, d)
    q, k = torch.empty((T, hq * d), dtype=td, device="cuda"), torch.empty((T, hk * d), dtype=td, device="cuda")
    ctx.qk_norm_rope_pwl(ctx.qk_rope_desc(qkv, hq, hk, d, q, positions=positions, cos_sin=cos_sin, gamma_q=g, gamma_k=g, pairs=pairs, k_out=k))
    v = qkv[:, (hq + hk) * d:].clone()
    ctx.qk_norm_rope_pwl(ctx.qk_rope_desc(qkv, hq, hk, d, qkv[:, :hq * d], positions=positions, cos_sin=cos_sin, gamma_q=g, gamma_k=g, pairs=pairs,
                                          k_out=qkv[:, hq * d:(hq + hk) * d]))
    ctx.check_device_status()
    assert torch.equal(qkv, torch.cat([q, k, v], 1))


def test_rope_bad_positions_and_slots_are_recorded_and_skipped(ctx):
    T, hq, hk, d, page, pages = 6, 2, 1, 64, 4, 3
    gen = gen_of(4)
    qkv = randn(gen, T, (hq + 2 * hk) * d)
    for bad in ("position", "slot"):
        positions, slots = i32([0, 1, 2, 3, 4, 5]), i32([0, 3, 11, 6, 7, 8])
        if bad == "position":
            positions[1], positions[2] = 10, -1
        else:
            slots[1], slots[2] = pages * page, 2 ** 31 - 1
        kc, vc = cache_views(torch.float32, pages, page, hk, d, "token", 7.0)
        q = torch.full((T, hq * d), 5.0, device="cuda")
        ctx.qk_norm_rope_pwl(ctx.qk_rope_desc(qkv, hq, hk, d, q, positions=positions, cos_sin=randn(gen, 10, d), k_cache=kc, v_cache=vc, slots=slots))
        assert ctx.poll_status() == 1
        assert (q[1:3] == 5).all() and not (q[[0, 3, 4, 5]] == 5).any()
        assert int((kc != 7).any(-1).sum()) == 4 and int((vc != 7).any(-1).sum()) == 4


# ---------------------------------------------------------------- attention


def make_cache(gen, td, lens, page, hk, d, layout, spare=2):
    """Pages in random order; every place that no token holds is NaN, table entries behind a row's pages are no page numbers."""
    used = [-(-n // page) for n in lens]
    pages, width = sum(used) + spare, max(used + [1]) + 1
    kc, vc = cache_views(td, pages, page, hk, d, layout, float("nan"))
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    tables = torch.full((len(lens), width + 3), -12345678, dtype=torch.int32, device="cuda")[:, :width]
    k, v, at = [], [], 0
    for i, n in enumerate(lens):
        tables[i, :used[i]] = order[at:at + used[i]]
        at += used[i]
        k.append(randn(gen, n, hk, d).to(td))
        v.append(randn(gen, n, hk, d).to(td))
        j = torch.arange(n, device="cuda")
        row = tables[i].long()[j // page]
        kc[row, j % page], vc[row, j % page] = k[-1], v[-1]
    return kc, vc, tables, k, v


P_STEP = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -16, torch.float16: 2.0 ** -21}


def check_attention(ctx, q, k, v, out, lens, hq, hk, d, td, scale=None):
    scale = np.float64(np.float32(d ** -0.5 if scale is None else scale))
    group = hq // hk
    qs, outs = f64(q), out
    for i, n in enumerate(lens):
        ki, vi = f64(k[i]), f64(v[i])
        want, bound = np.zeros((hq, d)), np.zeros((hq, d))
        for h in range(hq):
            want[h], bound[h] = ref.attention(qs[i, h], ki[:, h // group], vi[:, h // group], scale, ctx.tabs["exp"], ctx.tabs["recip"], P_STEP[td])
        # fp16 probabilities below its smallest normal number keep 2^-25 of 1, whatever their size
        if td == torch.float16 and n:
            bound += 2.0 ** -25 * np.abs(vi).sum(0).repeat(group, 0) * np.abs(ctx.tabs["recip"](1.0)[0])
        check(outs[i], want, bound, td, "request %d of %d tokens" % (i, n))


CASES = [
    # heads, key heads, d, page, lengths, layout
    (12, 12, 64, 16, [500], "token"), (12, 12, 64, 16, [1, 0, 2, 15, 16, 17, 33], "token"), (8, 1, 128, 16, [127, 128, 129, 1], "head"),
    (16, 2, 128, 64, [1000, 63, 64, 65], "both"), (20, 4, 64, 1, [5, 70], "token"), (6, 2, 96, 24, [0, 49, 300], "both"),
    (16, 1, 64, 128, [333, 1], "head"), (34, 2, 128, 8, [97, 9], "token"), (3, 3, 40, 5, [11, 260], "token"), (4, 2, 8, 32, [65], "token"),
    (10, 2, 256, 16, [40, 161], "both"), (7, 7, 128, 100, [900, 0, 0, 4], "head"), (4, 4, 248, 16, [30], "token"), (16, 16, 128, 16, [2600], "token"),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d,page,lens,layout", CASES)
def test_attention(ctx, dtype, hq, hk, d, page, lens, layout):
    td, gen, B = TYPES[dtype], gen_of(hq * d + page), len(lens)
    kc, vc, tables, k, v = make_cache(gen, td, lens, page, hk, d, layout)
    q = torch.full((B, 2 * hq + 1, d), float("nan"), dtype=td, device="cuda")[:, :hq]
    q.copy_(randn(gen, B, hq, d))
    raw = torch.full((B, hq * d + 16), 5.0, dtype=td, device="cuda")
    out = raw[:, :hq * d].view(B, hq, d)
    desc = ctx.attn_paged_desc(q, kc, vc, tables, i32(lens), out)
    ws = torch.full((ctx.attention_paged_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda")   # NaN throughout
    ctx.attention_pwl_paged(desc, ws)
    ctx.check_device_status()
    check_attention(ctx, q, k, v, out, lens, hq, hk, d, td)
    assert (raw[:, hq * d:] == 5).all()
    first = out.clone()
    ctx.attention_pwl_paged(desc, ws)
    ctx.check_device_status()
    assert torch.equal(out, first)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d", [(8, 1, 128), (2, 2, 64), (5, 1, 96)])
def test_attention_long_rows(ctx, dtype, hq, hk, d):
    """Many spans per row, and a row that is much shorter than the longest."""
    td, gen, lens = TYPES[dtype], gen_of(9), [20011, 130, 4096]
    kc, vc, tables, k, v = make_cache(gen, td, lens, 32, hk, d, "token")
    q = randn(gen, 3, hq, d).to(td)
    out = torch.empty_like(q)
    desc = ctx.attn_paged_desc(q, kc, vc, tables, i32(lens), out, max_len=20050)
    ctx.attention_pwl_paged(desc, torch.empty(ctx.attention_paged_workspace_bytes(desc), dtype=torch.uint8, device="cuda"))
    ctx.check_device_status()
    check_attention(ctx, q, k, v, out, lens, hq, hk, d, td)


def test_attention_offsets_beyond_31_bits(ctx):
    """A cache of more than 2^31 elements, its last page in use."""
    hq, hk, d, page, td = 8, 8, 128, 128, torch.bfloat16
    pages = (1 << 31) // (page * hk * d) + 2
    kc = torch.zeros((pages, page, hk, d), dtype=td, device="cuda")
    gen, n = gen_of(5), 200
    rows = [pages - 1, pages - 2]
    k, v = randn(gen, n, hk, d).to(td), randn(gen, n, hk, d).to(td)
    vc = torch.zeros_like(kc)
    for i, r in enumerate(rows):
        m = min(page, n - i * page)
        kc[r, :m], vc[r, :m] = k[i * page:i * page + m], v[i * page:i * page + m]
    q = randn(gen, 1, hq, d).to(td)
    out = torch.empty_like(q)
    desc = ctx.attn_paged_desc(q, kc, vc, i32([rows]), i32([n]), out)
    ctx.attention_pwl_paged(desc, torch.empty(ctx.attention_paged_workspace_bytes(desc), dtype=torch.uint8, device="cuda"))
    ctx.check_device_status()
    check_attention(ctx, q, [k], [v], out, [n], hq, hk, d, td)


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 64), ("bf16", 128), ("f16", 96)])
def test_attention_bad_pages_and_lengths_are_recorded(ctx, dtype, d):
    hq, hk, page, lens, td = 4, 2, 16, [40, 100, 20], TYPES[dtype]
    gen = gen_of(6)
    kc, vc, tables, k, v = make_cache(gen, td, lens, page, hk, d, "token")
    q = randn(gen, 3, hq, d).to(td)
    for what in ("page beyond", "page below", "length beyond", "length below"):
        t, n = tables.clone(), i32(lens)
        if "page" in what:
            t[1, 3] = kc.shape[0] if "beyond" in what else -1
        else:
            n[1] = 101 if "beyond" in what else -5
        out = torch.full_like(q, 5.0)
        desc = ctx.attn_paged_desc(q, kc, vc, t, n, out, max_len=100)
        ctx.attention_pwl_paged(desc, torch.empty(ctx.attention_paged_workspace_bytes(desc), dtype=torch.uint8, device="cuda"))
        assert ctx.poll_status() == (1 if "page" in what else 2)
        for i in (0, 2):
            check_attention(ctx, q[i:i + 1], [k[i]], [v[i]], out[i:i + 1], [lens[i]], hq, hk, d, td)
        if "length" in what:
            assert (out[1] == 5).all()


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128), ("f16", 64)])
def test_attention_nan_and_infinity_reach_their_heads_only(ctx, dtype, d):
    hq, hk, page, lens, td = 4, 2, 16, [40, 50], TYPES[dtype]
    gen = gen_of(8)
    kc, vc, tables, k, v = make_cache(gen, td, lens, page, hk, d, "token")
    vc[tables[0, 1].long(), 3, 0, 5] = float("inf")
    kc[tables[1, 2].long(), 1, 1, 7] = float("nan")
    q = randn(gen, 2, hq, d).to(td)
    out = torch.empty_like(q)
    desc = ctx.attn_paged_desc(q, kc, vc, tables, i32(lens), out)
    ctx.attention_pwl_paged(desc, torch.empty(ctx.attention_paged_workspace_bytes(desc), dtype=torch.uint8, device="cuda"))
    ctx.check_device_status()
    good = torch.isfinite(out)
    assert not good[0, :2, 5].any() and good[0, :2].sum() == 2 * (d - 1) and good[0, 2:].all()
    assert not good[1, 2:].any() and good[1, :2].all()


# ---------------------------------------------------------------- 4-bit linear


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,N,K,group,slot,residual,bias", [
    (1, 1, 32, 32, False, False, False), (1, 4096, 1024, 64, True, False, True), (2, 17, 128, 128, False, True, True), (7, 100, 416, 32, True, True, True),
    (8, 768, 768, 128, False, False, True), (9, 33, 4160, 64, False, False, False), (16, 64, 1152, 128, True, False, True),
    (17, 260, 96, 32, False, True, False), (32, 520, 2048, 64, False, False, True), (33, 40, 256, 128, True, True, True), (70, 300, 640, 32, False, True, True),
    (3, 5000, 160, 32, False, False, True), (1, 48, 8192, 128, False, True, True), (5, 16, 16448, 64, False, False, False)])
def test_linear_w4(nm, ctx, dtype, M, N, K, group, slot, residual, bias):
    td, gen = TYPES[dtype], gen_of(M * N + K)
    pad8 = lambda n: -(-n // 8) * 8  # noqa: E731
    a = torch.full((M, K + 8), float("nan"), dtype=td, device="cuda")[:, :K]
    a.copy_(randn(gen, M, K))
    codes = torch.randint(0, 256, (N, K // 2 + 16), generator=gen, device="cuda", dtype=torch.uint8)[:, :K // 2]
    scales = torch.full((N, K // group + 1), float("nan"), dtype=td, device="cuda")[:, :K // group]
    scales.copy_((0.1 * randn(gen, N, K // group) + 1) * 0.2 / K ** 0.5)
    b = 0.1 * randn(gen, N) if bias else None
    r = randn(gen, M, pad8(N)).to(td)[:, :N] if residual else None
    raw = torch.full((M, pad8(N) + 8), 5.0, dtype=td, device="cuda")
    ctx.linear_pwl_w4(ctx.linear_w4_desc(a, codes, scales, raw[:, :N], bias=b, residual=r, slot=nm.SLOT_GELU if slot else nm.SLOT_NONE))
    ctx.check_device_status()
    y, dy = ref.linear_w4(f64(a), codes.cpu().numpy(), f64(scales), None if b is None else f64(b), None if r is None else f64(r),
                          ctx.tabs["gelu"] if slot else None)
    check(raw[:, :N], y, dy, td)
    assert (raw[:, N:] == 5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_linear_w4_large_and_non_finite_activations(ctx, dtype):
    """Activations up to 2^120 (a group's sum before its scale has to stay finite), an infinity or NaN reaches its own token only."""
    td, M, N, K = TYPES[dtype], 4, 40, 256
    gen = gen_of(12)
    codes = torch.randint(0, 256, (N, K // 2), generator=gen, device="cuda", dtype=torch.uint8)
    scales = torch.full((N, 2), 2.0 ** -20, dtype=td, device="cuda")
    a = randn(gen, M, K).to(td)
    a[1] = 0
    a[1, 17] = min(torch.finfo(td).max, 2.0 ** 120)
    a[2, 100], a[3, 200] = float("nan"), float("inf")
    codes[:, 100] = 0x9b                                            # codes of 100's and 200's places are no zeros
    out = torch.empty((M, N), dtype=td, device="cuda")
    ctx.linear_pwl_w4(ctx.linear_w4_desc(a, codes, scales, out))
    ctx.check_device_status()
    y, dy = ref.linear_w4(f64(a[:2]), codes.cpu().numpy(), f64(scales), None, None, None)
    check(out[:2], y, dy, td)
    assert torch.isnan(out[2]).sum() >= N - 4 or torch.isnan(out[2]).all()
    assert torch.isinf(out[3]).all()


# ---------------------------------------------------------------- rows of every kind in one call


@pytest.mark.parametrize("dtype,hq,hk,d", [("bf16", 4, 1, 128), ("f16", 12, 1, 64), ("f32", 4, 2, 64), ("bf16", 3, 3, 40)])
def test_attention_many_short_rows_where_long_ones_may_come(ctx, dtype, hq, hk, d):
    """max_len says 20000, so the rows take equal shares; 300 of up to 200 tokens: several rows to a block, rows in two blocks, empty ones."""
    td, gen = TYPES[dtype], gen_of(31)
    lens = [int(n) for n in np.random.default_rng(5).integers(0, 201, 300)]
    lens[0] = lens[17] = lens[18] = lens[299] = 0
    lens[40] = 9000
    kc, vc, tables, k, v = make_cache(gen, td, lens, 32, hk, d, "token")
    wide = torch.full((300, 700), -5, dtype=torch.int32, device="cuda")
    wide[:, :tables.shape[1]] = tables
    q = randn(gen, 300, hq, d).to(td)
    out = torch.full_like(q, 5.0)
    desc = ctx.attn_paged_desc(q, kc, vc, wide, i32(lens), out, max_len=20000)
    ctx.attention_pwl_paged(desc, torch.full((ctx.attention_paged_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda"))
    ctx.check_device_status()
    some = [0, 1, 2, 17, 18, 39, 40, 41, 100, 255, 256, 257, 298, 299]
    for i in some:
        check_attention(ctx, q[i:i + 1], [k[i]], [v[i]], out[i:i + 1], [lens[i]], hq, hk, d, td)
    # every row alone gives what it gives among the others, up to the order of its sums
    assert torch.isfinite(out.float()).all() and not (out == 5).all(-1).any()


@pytest.mark.parametrize("dtype,hq,d", [("bf16", 4, 128), ("f16", 10, 64), ("f32", 3, 64), ("bf16", 2, 40)])
@pytest.mark.parametrize("requests", [1, 4, 5])
def test_attention_replayed_over_other_lengths(ctx, dtype, hq, d, requests):
    """A captured call over few long rows replayed as the lengths change: sums that an earlier replay left in the
    workspace are nobody's, a row that lay in many blocks may lie in one or have no token, a refused length leaves its output."""
    td, gen = TYPES[dtype], gen_of(requests)
    longest = [9001, 300, 4097, 64, 2500][:requests]
    kc, vc, tables, k, v = make_cache(gen, td, longest, 64, 1, d, "token")
    wide = torch.full((requests, 400), -5, dtype=torch.int32, device="cuda")
    wide[:, :tables.shape[1]] = tables
    q = randn(gen, requests, hq, d).to(td)
    out, lens = torch.full_like(q, 5.0), i32(longest)
    desc = ctx.attn_paged_desc(q, kc, vc, wide, lens, out, max_len=25000)
    ws = torch.full((ctx.attention_paged_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda")   # (with 40 channels none: one cluster)
    ctx.attention_pwl_paged(desc, ws)
    ctx.check_device_status()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        ctx.attention_pwl_paged(desc, ws)
    for change in (longest, [1] * requests, [0] * requests, [(n * 7) // 9 for n in longest], [25001] + longest[1:], longest):
        lens.copy_(i32(change))
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        refused = change[0] > 25000
        assert ctx.poll_status() == (2 if refused else 0)
        if refused:
            assert (out[0] == 5).all()
        for i in range(1 if refused else 0, requests):
            n = change[i]
            check_attention(ctx, q[i:i + 1], [k[i][:n]], [v[i][:n]], out[i:i + 1], [n], hq, 1, d, td)


@pytest.mark.parametrize("max_len", [0, 64, 20000])
def test_attention_of_empty_requests(ctx, max_len):
    q = randn(gen_of(1), 3, 4, 64).bfloat16()
    cache = torch.full((2, 16, 2, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 5.0)
    desc = ctx.attn_paged_desc(q, cache, cache, torch.full((3, 1250), -1, dtype=torch.int32, device="cuda"), i32([0, 0, 0]), out, max_len=max_len)
    ctx.attention_pwl_paged(desc, torch.empty(ctx.attention_paged_workspace_bytes(desc), dtype=torch.uint8, device="cuda"))
    ctx.check_device_status()
    assert (out == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_score_ranges(ctx, dtype):
    """Large scores of both signs: the maximum is the whole row's, whichever block, warp or lane has it, and values below the table's range
    take its first line."""
    hq, hk, d, td, n = 2, 1, 64, TYPES[dtype], 700
    gen = gen_of(77)
    for at in (0, 15, 16, 300, n - 1):
        kc, vc, tables, k, v = make_cache(gen, td, [n], 16, hk, d, "token")
        q = (4 * randn(gen, 1, hq, d)).to(td)
        k[0] *= 0.2
        k[0][at] = (q[0, 0] * 1.5).to(td)                      # far above all others for head 0
        j = torch.arange(n, device="cuda")
        row = tables[0].long()[j // 16]
        kc[row, j % 16] = k[0]
        out = torch.empty_like(q)
        desc = ctx.attn_paged_desc(q, kc, vc, tables, i32([n]), out)
        ctx.attention_pwl_paged(desc, torch.empty(ctx.attention_paged_workspace_bytes(desc), dtype=torch.uint8, device="cuda"))
        ctx.check_device_status()
        check_attention(ctx, q, k, v, out, [n], hq, hk, d, td)


def test_attention_two_calls_at_once(ctx):
    """Two streams, a workspace each, the form with equal shares: what each gives alone."""
    hq, hk, d, td, lens = 8, 2, 128, torch.bfloat16, [15000, 3000, 1, 12000]
    calls = []
    for seed in (1, 2):
        gen = gen_of(seed)
        kc, vc, tables, k, v = make_cache(gen, td, lens, 16, hk, d, "token")
        q = randn(gen, 4, hq, d).to(td)
        out = torch.empty_like(q)
        desc = ctx.attn_paged_desc(q, kc, vc, tables, i32(lens), out)
        calls.append((desc, torch.empty(ctx.attention_paged_workspace_bytes(desc), dtype=torch.uint8, device="cuda"), out))
    alone = []
    for desc, ws, out in calls:
        ctx.attention_pwl_paged(desc, ws)
        alone.append(out.clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for (desc, ws, out), s in zip(calls, streams):
            ctx.attention_pwl_paged(desc, ws, stream=s)
    torch.cuda.synchronize()
    ctx.check_device_status()
    for (_, _, out), want in zip(calls, alone):
        assert torch.equal(out, want)


# ---------------------------------------------------------------- a decoder's layer, step by step


class Layer:
    """Projection, head norms and rotation into the cache, attention, output projection of one layer with 4-bit weights, on arrays that
    stay the same from step to step, as a captured graph wants them."""

    def __init__(self, nm, ctx, seed, B, hq, hk, d, td, page=16, width=40, max_tokens=64):
        gen = gen_of(seed)
        H, rows = hq * d, (hq + 2 * hk) * d
        self.nm, self.ctx, self.B, self.hq, self.hk, self.d, self.td, self.page, self.H = nm, ctx, B, hq, hk, d, td, page, H
        pages = 3 * B + 60
        empty = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")  # noqa: E731
        self.lengths, self.new = torch.zeros(B, dtype=torch.int32, device="cuda"), empty(B)
        self.tables, self.free, self.count = torch.full((B, width), -1, dtype=torch.int32, device="cuda"), torch.randperm(pages, generator=gen, device="cuda").to(torch.int32), i32([pages])
        self.start, self.slots, self.positions = empty(B + 1), empty(max_tokens), empty(max_tokens)
        self.kc, self.vc = (torch.full((pages, page, hk, d), float("nan"), dtype=td, device="cuda") for _ in range(2))
        angle = torch.arange(width * page, device="cuda")[:, None] * 0.01 ** (torch.arange(d // 2, device="cuda") / (d // 2))
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float()
        self.gq, self.gk = 1 + 0.1 * randn(gen, d), 1 + 0.1 * randn(gen, d)
        weight = lambda n, k: (torch.randint(0, 256, (n, k // 2), generator=gen, device="cuda", dtype=torch.uint8),  # noqa: E731
                               ((1 + 0.1 * randn(gen, n, k // 64)) * 0.2 / k ** 0.5).to(td))
        self.wqkv, self.wo = weight(rows, H), weight(H, H)
        self.bias = 0.1 * randn(gen, rows)
        act = lambda n, w: torch.zeros((n, w), dtype=td, device="cuda")  # noqa: E731
        self.x, self.qkv, self.q, self.a, self.y = act(max_tokens, H), act(max_tokens, rows), act(max_tokens, H), act(B, H), act(B, H)
        self.plan = ctx.kv_plan_desc(self.lengths, self.new, self.tables, self.free, self.count, page, self.lengths, self.count, self.start, self.slots, self.positions)
        self.proj = ctx.linear_w4_desc(self.x, *self.wqkv, self.qkv, bias=self.bias)
        self.rope = ctx.qk_rope_desc(self.qkv, hq, hk, d, self.q, positions=self.positions, cos_sin=self.cos_sin, gamma_q=self.gq, gamma_k=self.gk,
                                     k_cache=self.kc, v_cache=self.vc, slots=self.slots)
        # (a step that adds one token to every request has them in the requests' order)
        self.attn = ctx.attn_paged_desc(self.q[:B].view(B, hq, d), self.kc, self.vc, self.tables, self.lengths, self.a.view(B, hq, d))
        self.ws = torch.empty(ctx.attention_paged_workspace_bytes(self.attn), dtype=torch.uint8, device="cuda")
        self.out = ctx.linear_w4_desc(self.a, *self.wo, self.y, residual=self.x[:B])

    def fill(self):
        """Prompts: keys and values of several tokens a request."""
        self.ctx.kv_plan(self.plan)
        self.ctx.linear_pwl_w4(self.proj)
        self.ctx.qk_norm_rope_pwl(self.rope)

    def step(self):
        self.fill()
        self.ctx.attention_pwl_paged(self.attn, self.ws)
        self.ctx.linear_pwl_w4(self.out)

    def state(self):
        return [t.clone() for t in (self.lengths, self.tables, self.free, self.count, self.start, self.slots, self.positions, self.kc.nan_to_num(7.0),
                                    self.vc.nan_to_num(7.0), self.qkv, self.q, self.a, self.y)]


@pytest.mark.parametrize("dtype,hq,hk,d", [("bf16", 4, 2, 64), ("f16", 8, 1, 128), ("f32", 2, 2, 64)])
def test_decoding_steps_eager_and_captured(nm, ctx, dtype, hq, hk, d):
    td, B = TYPES[dtype], 6
    eager, graphed = (Layer(nm, ctx, 9, B, hq, hk, d, td) for _ in range(2))
    prompts = [5, 16, 1, 20, 13, 9]
    for layer in (eager, graphed):
        layer.new.copy_(i32(prompts))
        layer.x.copy_(randn(gen_of(50), *layer.x.shape))
        layer.fill()
    assert eager.lengths.tolist() == prompts
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphed.new.fill_(1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):   # the calls go to the capturing stream
        graphed.step()
    for n in range(20):
        new = [1] * B
        if n == 7:
            new[3] = -1                          # request 3 ends ...
        if n == 8:
            new[3] = 1                           # ... and another one takes its place
        for layer in (eager, graphed):
            layer.new.copy_(i32(new))
            layer.x.copy_(randn(gen_of(100 + n), *layer.x.shape))
        if n == 7:                               # tokens and requests are not one to one in this step: the cache alone is filled
            eager.fill(), graphed.fill()
        else:
            eager.step()
            graph.replay()
        torch.cuda.synchronize()
        ctx.check_device_status()
        for s, t in zip(eager.state(), graphed.state()):
            assert torch.equal(s, t), n
    # the last step stage by stage, each from what the one before it has left
    L, T = eager, B
    y, dy = ref.linear_w4(f64(L.x), L.wqkv[0].cpu().numpy(), f64(L.wqkv[1]), f64(L.bias), None, None)
    check(L.qkv, y, dy, td, "projection")
    x, pos = f64(L.qkv).reshape(-1, hq + 2 * hk, d)[:T], L.positions.cpu().numpy()[:T]
    assert pos.tolist() == [n - 1 for n in L.lengths.tolist()]
    q, dq = ref.rope(x[:, :hq], pos, f64(L.cos_sin), f64(L.gq), 1e-6, d, False, ctx.tabs["rsqrt"])
    check(L.q[:T], q.reshape(T, -1), dq.reshape(T, -1), td, "queries")
    k, dk = ref.rope(x[:, hq:hq + hk], pos, f64(L.cos_sin), f64(L.gk), 1e-6, d, False, ctx.tabs["rsqrt"])
    at = L.slots[:T].long()
    check(L.kc[at // 16, at % 16], k, dk, td, "keys")
    lens = L.lengths.tolist()
    rows = [L.tables[i].long()[torch.arange(n, device="cuda") // 16] for i, n in enumerate(lens)]
    place = [torch.arange(n, device="cuda") % 16 for n in lens]
    check_attention(ctx, L.q[:T].view(T, hq, d), [L.kc[r, p] for r, p in zip(rows, place)], [L.vc[r, p] for r, p in zip(rows, place)], L.a.view(T, hq, d), lens, hq,
                    hk, d, td)
    y, dy = ref.linear_w4(f64(L.a), L.wo[0].cpu().numpy(), f64(L.wo[1]), None, f64(L.x[:B]), None)
    check(L.y, y, dy, td, "output")
    assert len(set(torch.cat(rows).tolist())) == sum(-(-n // 16) for n in lens)   # no page has two owners
