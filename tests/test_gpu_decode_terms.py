"""GPU tests of the digits that the decoding operators keep: inputs whose sums nearly cancel, or lie in many small terms."""
import numpy as np
import pytest
import torch

import decode_ref as ref
from decode_ref import HALF_STEP, TYPES, U, check, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(nm):
    c = nm.Context(0)
    c.tabs = ref.load_tables(c)
    yield c
    c.close()


def table32(tab, x):
    """The table as fp32 evaluates it, bit for bit: one FMA, the segment from (x - lo) n / (hi - lo), which is exact for the scores used here."""
    s = np.clip(np.floor((x - tab.lo) * tab.n / (tab.hi - tab.lo)), 0, tab.n - 1).astype(int)
    return (tab.k[s] * x + tab.b[s]).astype(np.float32).astype(np.float64)


def attend(ctx, q, k, v, max_len, page=16):
    """One request, one key head: q [heads, d], k, v [n, d], the scores as they are (scale 1)."""
    n, d = k.shape
    pages = -(-n // page)
    kc, vc = (torch.full((pages, page, 1, d), float("nan"), dtype=q.dtype, device="cuda") for _ in range(2))
    kc.view(-1, d)[:n], vc.view(-1, d)[:n] = k, v
    table = torch.full((1, -(-max_len // page)), -1, dtype=torch.int32, device="cuda")
    table[0, :pages] = torch.arange(pages, device="cuda")
    out = torch.empty_like(q)[None]
    desc = ctx.attn_paged_desc(q[None].contiguous(), kc, vc, table, torch.tensor([n], dtype=torch.int32, device="cuda"), out, max_len=max_len, scale=1.0)
    ctx.attention_pwl_paged(desc, torch.full((ctx.attention_paged_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda"))
    ctx.check_device_status()
    return out[0]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("below", [(15.4, 15.5), (15.8, 16.2)])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_many_small_probabilities(ctx, dtype, below, d):
    """One token far above 131070 others, which have 1e-7 of its weight each and some hundredths of it together: rounded on fp16's grid of 2^-24
    each would be off by up to a quarter, on one side."""
    td, n = TYPES[dtype], 131071
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d)
    s = -(below[0] + (below[1] - below[0]) * torch.rand(n, generator=gen, device="cuda")).to(td)
    s[777] = 0
    k = torch.zeros((n, d), dtype=td, device="cuda")
    k[:, 3] = s
    v = (0.5 + torch.rand((n, d), generator=gen, device="cuda")).to(td)
    q = torch.zeros((2, d), dtype=td, device="cuda")
    q[0, 3] = q[1, 3] = 1
    out = attend(ctx, q, k, v, n, page=64)
    e, vv = table32(ctx.tabs["exp"], f64(s)), f64(v)
    # A term passes through at most: a product's sum and a warp's tiles (some 450 tokens a block), 8 warps, 296 blocks; 512 roundings cover them.
    depth = 512 * U
    r, dr = ctx.tabs["recip"](e.sum(), depth * e.sum())
    o = e @ vv
    check(out, np.stack([o * r] * 2), np.stack([o * dr + depth * o * (r + dr)] * 2), td)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("max_len", [16, 20000])   # one launch, shares of tokens
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_attention_probabilities_keep_24_bits(ctx, dtype, max_len, d):
    """Per head, three tokens of the highest score whose values add up to the probability of a fourth, which has the value -1: what is left
    shows 2^-20 of a probability.  The fourth's scores are those whose probability two terms of bf16 would miss most."""
    td, heads = TYPES[dtype], 8
    grid = torch.linspace(-3, -0.05, 4000).to(td).unique().double().numpy()
    e = table32(ctx.tabs["exp"], grid)
    two = lambda x: x - x.float().bfloat16().double()  # noqa: E731
    missed = (two(two(torch.from_numpy(e))).abs() / torch.from_numpy(e)).numpy()
    pick = np.argsort(-missed)[:heads]
    assert missed[pick].min() > 40 * U
    e0, e3 = table32(ctx.tabs["exp"], np.zeros(1))[0], e[pick]
    q, k, v = (torch.zeros(s, dtype=td, device="cuda") for s in ((heads, d), (4, d), (4, d)))
    for h in range(heads):
        q[h, h] = 1
        k[3, h] = float(grid[pick[h]])
        rest = e3[h] / e0
        for j in range(3):
            v[j, h] = rest
            rest -= float(v[j, h])
    v[3] = -1
    out = f64(attend(ctx, q, k, v, max_len))
    vv = f64(v)
    for h in range(heads):
        w = np.array([e0, e0, e0, e3[h]])
        o, size = w @ vv[:, h], w @ np.abs(vv[:, h])
        r, dr = ctx.tabs["recip"](w.sum(), 8 * U * w.sum())
        # the tile's sum: five numbers at most, each cut at 2^-24 of the largest, some three times; nothing is added to it but zeros
        bound = 15 * U * size * (r + dr) + abs(o) * dr
        assert abs(out[h, h] - o * r) <= bound + (abs(o * r) + bound) * HALF_STEP[td] + 2.0 ** -25, (h, out[h, h], o * r)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("max_len", [100, 20000])
@pytest.mark.parametrize("d", [64, 128, 40])
def test_attention_infinite_values_give_infinities(ctx, dtype, max_len, d):
    """Every probability is positive, so a channel with an infinite value of one sign is infinite, in each head."""
    td, n, heads = TYPES[dtype], 90, 6
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d)
    q = 0.3 * torch.randn((heads, d), generator=gen, device="cuda")
    k, v = torch.randn((n, d), generator=gen, device="cuda"), torch.randn((n, d), generator=gen, device="cuda")
    v[torch.arange(0, 40), 5] = float("inf")
    v[41, 6], v[89, 7] = float("-inf"), float("inf")
    v[3, 8], v[4, 8] = float("inf"), float("-inf")
    out = attend(ctx, q.to(td), k.to(td), v.to(td), max_len).float()
    assert (out[:, 5] == float("inf")).all() and (out[:, 6] == float("-inf")).all() and (out[:, 7] == float("inf")).all()
    assert torch.isnan(out[:, 8]).all()
    rest = torch.ones(d, dtype=torch.bool, device="cuda")
    rest[5:9] = False
    assert torch.isfinite(out[:, rest]).all()


@pytest.mark.parametrize("M", [1, 8, 9, 17, 32])
@pytest.mark.parametrize("K,group", [(128, 128), (128, 64), (96, 32), (1024, 128)])
def test_linear_w4_fp32_sums_are_not_cut(ctx, M, K, group):
    """fp32 activations and weights of one sign, where truncated sums are all short: on average nearly nothing is missing.  The tensor core loses
    1.55e-8 of a sum per step (a quarter of 2^-24); two such steps per 32 k count here, less than half of 2^-24 on average, and roundings to
    nearest have no preferred sign."""
    N = 4096
    gen = torch.Generator(device="cuda")
    gen.manual_seed(M * K + group)
    a = 1 + torch.rand((M, K), generator=gen, device="cuda")
    codes = torch.randint(9, 16, (N, K // 2, 2), generator=gen, device="cuda", dtype=torch.uint8)
    codes = codes[..., 0] | codes[..., 1] << 4
    scales = torch.ones((N, K // group), device="cuda")
    out = torch.empty((M, N), device="cuda")
    ctx.linear_pwl_w4(ctx.linear_w4_desc(a, codes, scales, out))
    ctx.check_device_status()
    y, _ = ref.linear_w4(f64(a), codes.cpu().numpy(), f64(scales), None, None, None)
    off = (f64(out) - y) / y
    assert abs(off.mean()) <= U, off.mean() / U
    # the largest: K / 32 additions of a token's steps and some of warps, half a unit each, and the two truncations
    assert np.abs(off).max() <= (K / 32 + 8) * U, np.abs(off).max() / U
