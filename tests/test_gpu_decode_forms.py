"""GPU tests of the decoding operators in the forms and combinations that their neighbours' tests leave out."""
import numpy as np
import pytest
import torch

import decode_ref as ref
from decode_ref import TYPES, check, f64
from test_gpu_decode import Layer, check_attention, ctx, gen_of, i32, make_cache, randn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hk", [(0, 2), (3, 0)])
def test_rope_gamma_of_no_heads(ctx, dtype, hq, hk):  # noqa: F811
    """A gamma for heads that are not there, with a slot that holds no table: nothing is normed."""
    td, gen, T, d = TYPES[dtype], gen_of(hq), 9, 64
    qkv = randn(gen, T, (hq + 2 * hk) * d).to(td)
    g = 1 + 0.1 * randn(gen, d)
    q, k = torch.full((T, hq * d), 5.0, dtype=td, device="cuda"), torch.full((T, hk * d), 5.0, dtype=td, device="cuda")
    ctx.qk_norm_rope_pwl(ctx.qk_rope_desc(qkv, hq, hk, d, q, gamma_q=None if hq else g, gamma_k=None if hk else g, k_out=k, rsqrt_slot=15))
    ctx.check_device_status()
    assert torch.equal(q, qkv[:, :hq * d]) and torch.equal(k, qkv[:, hq * d:(hq + hk) * d])


# ---------------------------------------------------------------- the rows of a plan


@pytest.mark.parametrize("dtype,hq,hk,d", [("bf16", 8, 2, 64), ("f16", 4, 1, 128), ("f32", 6, 2, 64), ("bf16", 3, 3, 40)])
@pytest.mark.parametrize("max_len,B", [(300, 7), (20000, 7), (20000, 2)])   # one launch, shares of tokens, a third launch where units are few
def test_attention_finds_its_rows_in_a_plan(ctx, dtype, hq, hk, d, max_len, B):  # noqa: F811
    """Requests with one new token, several, or none (in use, over, never there): each query and output at its last new token's row; nothing
    is read or written for a request without one."""
    td, gen = TYPES[dtype], gen_of(B + d)
    lens = [129, 300, 40, 0, 17, 250, 64][:B]
    new = [1, 3, 0, 0, 5, 0, 2][:B] if B > 2 else [0, 2]
    start = np.concatenate([[0], np.cumsum(new)])
    rows = int(start[-1]) + 4
    kc, vc, tables, k, v = make_cache(gen, td, lens, 32, hk, d, "token")
    wide = torch.full((B, 700), -5, dtype=torch.int32, device="cuda")
    wide[:, :tables.shape[1]] = tables
    lengths = i32(lens)
    for b in range(B):
        if new[b] == 0:
            wide[b], lengths[b] = -7, [max_len, max_len + 1, -3][b % 3]
    q = torch.full((rows, hq + 1, d), float("nan"), dtype=td, device="cuda")[:, :hq]
    last = [int(start[b + 1]) - 1 for b in range(B) if new[b]]
    q[last] = randn(gen, len(last), hq, d).to(td)
    raw = torch.full((rows, hq * d + 8), 5.0, dtype=td, device="cuda")
    out = raw[:, :hq * d].view(rows, hq, d)
    desc = ctx.attn_paged_desc(q, kc, vc, wide, lengths, out, max_len=max_len, token_start=i32(start.tolist()))
    ctx.attention_pwl_paged(desc, torch.full((ctx.attention_paged_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda"))
    ctx.check_device_status()
    for b in range(B):
        if new[b]:
            at = slice(int(start[b + 1]) - 1, int(start[b + 1]))
            check_attention(ctx, q[at], [k[b]], [v[b]], out[at], [lens[b]], hq, hk, d, td)
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[last] = False
    assert (out[rest] == 5).all() and (raw[:, hq * d:] == 5).all()


@pytest.mark.parametrize("max_len", [300, 20000])
def test_attention_refuses_rows_that_are_none(ctx, max_len):  # noqa: F811
    hq, hk, d, td, lens, rows = 4, 2, 64, torch.bfloat16, [30, 70, 0, 20], 4
    gen = gen_of(12)
    kc, vc, tables, k, v = make_cache(gen, td, lens, 32, hk, d, "token")
    wide = torch.full((4, 700), -5, dtype=torch.int32, device="cuda")
    wide[:, :tables.shape[1]] = tables
    q = randn(gen, rows, hq, d).to(td)
    # (start, requests left out, status)
    for start, left_out, status in (([0, 1, 2, 3, 4], [], 0), ([0, 1, 5, 5, 5], [1, 2, 3], 1), ([0, 1, 0, 2, 3], [1], 1), ([0, 1, -1, 3, 4], [1, 2], 1),
                                    ([-2, -1, 2, 3, 4], [0, 1], 1), ([0, 0, 0, 0, 0], [0, 1, 2, 3], 0), ([0, 1, 2 ** 31 - 1, -2 ** 31, 4], [1, 2, 3], 1)):
        out = torch.full_like(q, 5.0)
        desc = ctx.attn_paged_desc(q, kc, vc, wide, i32(lens), out, max_len=max_len, token_start=i32(start))
        ctx.attention_pwl_paged(desc, torch.empty(ctx.attention_paged_workspace_bytes(desc), dtype=torch.uint8, device="cuda"))
        assert ctx.poll_status() == status, start
        done = [b for b in range(4) if b not in left_out and start[b + 1] > start[b]]
        for b in done:
            r = start[b + 1] - 1
            check_attention(ctx, q[r:r + 1], [k[b]], [v[b]], out[r:r + 1], [lens[b]], hq, hk, d, td)
        rest = [r for r in range(rows) if r not in [start[b + 1] - 1 for b in done]]
        assert (out[rest] == 5).all(), start


class PackedLayer(Layer):
    """A layer whose rows are the step's new tokens, however many each request has."""

    def __init__(self, nm, ctx, seed, B, hq, hk, d, td, max_tokens=64):  # noqa: F811
        super().__init__(nm, ctx, seed, B, hq, hk, d, td, max_tokens=max_tokens)
        self.a, self.y = (torch.zeros((max_tokens, self.H), dtype=td, device="cuda") for _ in range(2))
        self.attn = ctx.attn_paged_desc(self.q.view(max_tokens, hq, d), self.kc, self.vc, self.tables, self.lengths, self.a.view(max_tokens, hq, d),
                                        token_start=self.start)
        self.ws = torch.empty(ctx.attention_paged_workspace_bytes(self.attn), dtype=torch.uint8, device="cuda")
        self.out = ctx.linear_w4_desc(self.a, *self.wo, self.y, residual=self.x)


@pytest.mark.parametrize("dtype,hq,hk,d", [("bf16", 4, 2, 64), ("f16", 8, 1, 128), ("f32", 2, 2, 64)])
def test_decoding_steps_in_which_requests_idle_end_and_join(nm, ctx, dtype, hq, hk, d):  # noqa: F811
    """Plan, projection, rotation, attention, projection, eager and replayed, over steps of every kind; after each step every request's
    attention is that of its own query, and what the step did not touch is as it was."""
    td, B = TYPES[dtype], 6
    eager, graphed = (PackedLayer(nm, ctx, 9, B, hq, hk, d, td) for _ in range(2))
    for layer in (eager, graphed):
        layer.new.copy_(i32([5, 16, 0, 20, 1, 0]))
        layer.x.copy_(randn(gen_of(50), *layer.x.shape))
        layer.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        graphed.step()
    steps = [[1, 1, 1, 1, 1, 1], [1, 0, 1, 1, 0, 1], [1, -1, 1, 1, 1, 1], [1, 9, 0, -1, 1, 1], [0, 0, 0, 0, 0, 0], [-1, 1, 1, 4, -1, 1], [30, 1, -1, 1, 20, 0],
             [1, 1, 0, 1, 1, 1], [60, 1, 1, 1, 1, 1]]
    for n, new in enumerate(steps):
        before = eager.a.clone()
        for layer in (eager, graphed):
            layer.new.copy_(i32(new))
            layer.x.copy_(randn(gen_of(100 + n), *layer.x.shape))
        eager.step()
        graph.replay()
        torch.cuda.synchronize()
        status = 2 if sum(max(x, 0) for x in new) > 64 else 0     # the last step has more tokens than rows: it is left out whole
        assert ctx.poll_status() == status
        for s, t in zip(eager.state(), graphed.state()):
            assert torch.equal(s, t), n
        start, lens, T = eager.start.tolist(), eager.lengths.tolist(), eager.q.shape[0]
        touched = []
        for b in range(B):
            if status or new[b] <= 0:
                assert start[b + 1] == start[b]
                continue
            r = start[b + 1] - 1
            touched.append(r)
            j = torch.arange(lens[b], device="cuda")
            row = eager.tables[b].long()[j // eager.page]
            assert int(eager.positions[r]) == lens[b] - 1
            check_attention(ctx, eager.q.view(T, hq, d)[r:r + 1], [eager.kc[row, j % eager.page]], [eager.vc[row, j % eager.page]],
                            eager.a.view(T, hq, d)[r:r + 1], [lens[b]], hq, hk, d, td)
        rest = [r for r in range(T) if r not in touched]
        assert torch.equal(eager.a[rest], before[rest]), n
        y, dy = ref.linear_w4(f64(eager.a), eager.wo[0].cpu().numpy(), f64(eager.wo[1]), None, f64(eager.x), None)
        check(eager.y, y, dy, td, "output")


# ---------------------------------------------------------------- a reciprocal for rows of every length


RECIP_1_2 = 12   # a slot of its own: the other tests' tables stay


class Pow2:
    """A table over [1, 2] applied to mantissas: the lines of both ends meet at powers of two, up to their rounding."""

    def __init__(self, tab):
        self.tab = tab

    def __call__(self, x, err=0.0):
        p = 2.0 ** -np.floor(np.log2(x))
        r, dr = self.tab(x * p, err * p)
        return r * p, (dr + 8 * ref.U) * p


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("hq,d", [(1, 64), (12, 64), (4, 40), (2, 128)])
@pytest.mark.parametrize("max_len,lens", [(600, [1, 3, 16, 100, 600, 0, 2]), (9000, [1, 16, 9000, 4097, 100]), (20000, [20000, 1]), (20000, [1, 30, 999, 7, 0, 2048])])
def test_attention_is_a_softmax_for_every_length(nm, ctx, dtype, hq, d, max_len, lens):  # noqa: F811
    """One reciprocal table on [1, 2] for all rows of a call, with recip_pow2."""
    ctx.load_function_table(RECIP_1_2, nm.FUNC_RECIP, 256, 1.0, 2.0)
    tab = Pow2(ref.Table(nm.FUNC_RECIP, 256, 1.0, 2.0))
    td, gen, B = TYPES[dtype], gen_of(len(lens) + d), len(lens)
    kc, vc, tables, k, v = make_cache(gen, td, lens, 32, 1, d, "token")
    wide = torch.full((B, -(-max_len // 32)), -5, dtype=torch.int32, device="cuda")
    width = min(wide.shape[1], tables.shape[1])
    wide[:, :width] = tables[:, :width]
    q = randn(gen, B, hq, d).to(td)
    out = torch.full_like(q, 5.0)
    desc = ctx.attn_paged_desc(q, kc, vc, wide, i32(lens), out, max_len=max_len, recip_slot=RECIP_1_2, recip_pow2=True)
    ctx.attention_pwl_paged(desc, torch.full((ctx.attention_paged_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda"))
    ctx.check_device_status()
    scale = np.float64(np.float32(d ** -0.5))
    for i, n in enumerate(lens):
        ki, vi = f64(k[i])[:, 0], f64(v[i])[:, 0]
        want, bound, soft, far = (np.zeros((hq, d)) for _ in range(4))
        for h in range(hq if n else 0):
            want[h], bound[h] = ref.attention(f64(q)[i, h], ki, vi, scale, ctx.tabs["exp"], tab, 0.0)
            s = scale * (ki @ f64(q)[i, h])
            p = np.exp(s - s.max())
            p /= p.sum()
            # secants of exp over 1/16 lie up to (1/16)^2 / 8 above it, of 1/x over 1/256 up to 2 (1/256)^2 / 8 above it; a weight's numerator and
            # the sum both have the first
            soft[h], far[h] = p @ vi, (2 * (1 / 16) ** 2 / 8 + 2 * (1 / 256) ** 2 / 8) * (p @ np.abs(vi))
        check(out[i], want, bound, td, "request %d of %d tokens" % (i, n))
        check(out[i], soft, bound + far, td, "softmax of %d tokens" % n)


def test_attention_weights_add_up_to_one(nm, ctx):  # noqa: F811
    """Values of one: what comes out is the sum of the weights, 1 with recip_pow2; with one table over all sums far from it."""
    ctx.load_function_table(RECIP_1_2, nm.FUNC_RECIP, 256, 1.0, 2.0)
    ctx.load_function_table(13, nm.FUNC_RECIP, 256, 32.0, 8193.0)
    lens, hq, d = [1, 2, 16, 100, 1000, 8192], 4, 64
    gen = gen_of(3)
    kc, vc, tables, k, v = make_cache(gen, torch.float32, lens, 64, 2, d, "token")
    vc.fill_(1.0)
    q = randn(gen, len(lens), hq, d)
    out = torch.empty_like(q)
    for slot, pow2 in ((RECIP_1_2, True), (13, False)):
        desc = ctx.attn_paged_desc(q, kc, vc, tables, i32(lens), out, max_len=8192, recip_slot=slot, recip_pow2=pow2)
        ctx.attention_pwl_paged(desc, torch.empty(ctx.attention_paged_workspace_bytes(desc), dtype=torch.uint8, device="cuda"))
        ctx.check_device_status()
        off = (out.double() - 1).abs().amax((1, 2)).tolist()
        if pow2:   # 2 (1/256)^2 / 8 of the table; two sums of n terms in some order of at most 300 steps each
            assert max(off) <= 2 * (1 / 256) ** 2 / 8 + 600 * 2.0 ** -24, off
        else:
            assert off[0] > 0.9 and off[-1] < 0.1, off


# ---------------------------------------------------------------- equal shares of all tokens: what the one-launch form is tested for


def shares(ctx, q, kc, vc, tables, lens, out=None, max_len=20000, **kw):  # noqa: F811
    """The call with room for max_len tokens a request, so that blocks take equal shares; a workspace of NaN."""
    wide = torch.full((len(lens), -(-max_len // kc.shape[1])), -5, dtype=torch.int32, device="cuda")
    width = min(wide.shape[1], tables.shape[1])
    wide[:, :width] = tables[:, :width]
    out = torch.full_like(q, 5.0) if out is None else out
    desc = ctx.attn_paged_desc(q, kc, vc, wide, i32(lens), out, max_len=max_len, **kw)
    need = ctx.attention_paged_workspace_bytes(desc)
    assert need > 0
    ctx.attention_pwl_paged(desc, torch.full((need,), 255, dtype=torch.uint8, device="cuda"))
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d,layout", [(4, 2, 256, "token"), (9, 1, 256, "both"), (16, 1, 96, "head"), (16, 1, 128, "token"), (40, 2, 128, "token"),
                                            (20, 1, 64, "both"), (6, 2, 200, "head"), (2, 1, 8, "token")])
def test_attention_shares_of_every_core(ctx, dtype, hq, hk, d, layout):  # noqa: F811
    """256 channels (one block an SM, two pieces a lane in fp32), 16 query heads a unit, odd head sizes."""
    td, gen, lens = TYPES[dtype], gen_of(hq + d), [1700, 0, 33, 5003, 1]
    kc, vc, tables, k, v = make_cache(gen, td, lens, 24, hk, d, layout)
    q = randn(gen, len(lens), hq, d).to(td)
    out = shares(ctx, q, kc, vc, tables, lens, max_len=100008 if d in (8, 200) else 20000)
    ctx.check_device_status()
    check_attention(ctx, q, k, v, out, lens, hq, hk, d, td)


@pytest.mark.parametrize("dtype,hq,hk,d", [("bf16", 4, 1, 128), ("f16", 12, 1, 64), ("f32", 4, 2, 64)])
def test_attention_shares_every_row_of_many(ctx, dtype, hq, hk, d):  # noqa: F811
    td, gen = TYPES[dtype], gen_of(32)
    lens = [int(n) for n in np.random.default_rng(6).integers(0, 161, 300)]
    lens[0] = lens[17] = lens[18] = lens[299] = 0
    lens[40], lens[41], lens[42] = 3001, 32, 31
    kc, vc, tables, k, v = make_cache(gen, td, lens, 32, hk, d, "token")
    q = randn(gen, 300, hq, d).to(td)
    out = shares(ctx, q, kc, vc, tables, lens)
    ctx.check_device_status()
    check_attention(ctx, q, k, v, out, lens, hq, hk, d, td)


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128), ("f16", 64), ("bf16", 40)])
@pytest.mark.parametrize("requests", [1, 3])   # with one request few units, joined by a third launch
def test_attention_shares_nan_and_infinity_reach_their_heads_only(ctx, dtype, d, requests):  # noqa: F811
    hq, hk, lens, td = 4, 2, [4000, 5000, 70][:requests], TYPES[dtype]
    gen = gen_of(8)
    kc, vc, tables, k, v = make_cache(gen, td, lens, 16, hk, d, "token")
    vc[tables[0, 201].long(), 3, 0, 5] = float("inf")
    kc[tables[requests - 1, 2].long(), 1, 1, 7] = float("nan")
    q = randn(gen, requests, hq, d).to(td)
    out = shares(ctx, q, kc, vc, tables, lens, max_len=100000)
    ctx.check_device_status()
    good = torch.isfinite(out)
    assert not good[0, :2, 5].any() and good[0, :2].sum() == 2 * (d - 1)
    assert not good[requests - 1, 2:].any()
    if requests > 1:
        assert good[0, 2:].all() and good[1].all() and good[2, :2].all()
        check_attention(ctx, q[1:2], k[1:2], v[1:2], out[1:2], lens[1:2], hq, hk, d, td)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_shares_offsets_beyond_31_bits(ctx, dtype):  # noqa: F811
    """A cache of more than 2^31 elements, its last pages in use."""
    hq, hk, d, page, td, n = 8, 8, 128, 128, TYPES[dtype], 300
    pages = (1 << 31) // (page * hk * d) + 3
    kc, vc = (torch.zeros((pages, page, hk, d), dtype=td, device="cuda") for _ in range(2))
    gen = gen_of(5)
    rows = [pages - 1, 0, pages - 2]
    k, v = randn(gen, n, hk, d).to(td), randn(gen, n, hk, d).to(td)
    for i, r in enumerate(rows):
        m = min(page, n - i * page)
        kc[r, :m], vc[r, :m] = k[i * page:i * page + m], v[i * page:i * page + m]
    q = randn(gen, 1, hq, d).to(td)
    out = shares(ctx, q, kc, vc, i32([rows]), [n])
    ctx.check_device_status()
    check_attention(ctx, q, [k], [v], out, [n], hq, hk, d, td)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M", [3, 12, 32])
def test_linear_w4_nan_reaches_its_token_and_all_of_it(ctx, dtype, M):  # noqa: F811
    """A NaN times any code is NaN, of a code of zero too; the other tokens' sums are as without it."""
    td, N, K = TYPES[dtype], 72, 512
    gen = gen_of(M)
    codes = torch.randint(0, 256, (N, K // 2), generator=gen, device="cuda", dtype=torch.uint8)
    scales = torch.full((N, K // 128), 0.25, dtype=td, device="cuda")
    a = randn(gen, M, K).to(td)
    a[1, 301], a[M - 1, 5] = float("nan"), float("inf")
    codes[:, 2] = 0x98                                     # the infinity meets a code of one (the high half), and its neighbour one of zero
    out = torch.empty((M, N), dtype=td, device="cuda")
    ctx.linear_pwl_w4(ctx.linear_w4_desc(a, codes, scales, out))
    ctx.check_device_status()
    assert torch.isnan(out[1]).all() and (out[M - 1] == float("inf")).all()
    rest = [m for m in range(M) if m not in (1, M - 1)]
    y, dy = ref.linear_w4(f64(a[rest]), codes.cpu().numpy(), f64(scales), None, None, None)
    check(out[rest], y, dy, td)
