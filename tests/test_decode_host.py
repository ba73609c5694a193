"""CPU-only checks of the decoding operators: what their entry points and the binding refuse, and the reference plan."""
import ctypes as C

import numpy as np
import pytest
import torch

import decode_ref as ref
import paper_2305_14405_b200 as nm


@pytest.fixture(scope="module")
def lib():
    from paper_2305_14405_b200 import build
    build.build()
    return nm.load()


@pytest.fixture(scope="module")
def ctx(lib):
    """A context that no device backs: enough for calls that are refused before anything is launched."""
    if torch.cuda.is_available():
        pytest.skip("a machine without a device")
    buf = C.create_string_buffer(1 << 17)
    k = (C.c_float * 4)()
    for slot in (nm.SLOT_GELU, nm.SLOT_EXP, nm.SLOT_RECIP, nm.SLOT_RSQRT):
        assert lib.nm_pwl_table_load(buf, slot, 4, 0.0, 1.0, k, k) == 6   # the host side of the table; there is no device to copy it to
    return buf


A = 1 << 20     # an aligned address that is never followed


def plan_desc(**kw):
    d = nm.KvPlanDesc()
    d.B, d.page_size, d.max_pages, d.max_tokens, d.free_capacity, d.ld_tables = 2, 16, 4, 8, 32, 4
    for name in ("lengths", "new_tokens", "free_count", "block_tables", "free_pages", "lengths_out", "free_count_out", "token_start", "slots", "positions"):
        setattr(d, name, A)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def rope_desc(**kw):
    d = nm.QkRopeDesc()
    d.T, d.heads, d.kv_heads, d.d, d.rot, d.dtype = 3, 4, 2, 64, 32, nm.BF16
    d.ld_qkv, d.ld_q, d.ld_k, d.max_position, d.eps, d.rsqrt_slot = 512, 256, 128, 100, 1e-6, nm.SLOT_RSQRT
    d.num_pages, d.page_size, d.stride_page, d.stride_token, d.stride_head = 8, 16, 2048, 128, 64
    for name in ("qkv", "positions", "cos_sin", "gamma_q", "gamma_k", "q_out", "k_out", "k_cache", "v_cache", "slots"):
        setattr(d, name, A)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def attn_desc(**kw):
    d = nm.AttnPagedDesc()
    d.B, d.heads, d.kv_heads, d.d, d.dtype, d.num_pages, d.page_size, d.max_pages, d.max_len = 2, 8, 2, 64, nm.F16, 9, 16, 4, 64
    d.ld_q, d.ld_out, d.ld_tables, d.stride_page, d.stride_token, d.stride_head = 512, 512, 4, 2048, 128, 64
    d.scale, d.exp_slot, d.recip_slot = 0.125, nm.SLOT_EXP, nm.SLOT_RECIP
    for name in ("Q", "k_cache", "v_cache", "block_tables", "lengths", "out"):
        setattr(d, name, A)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def w4_desc(**kw):
    d = nm.LinearW4Desc()
    d.M, d.N, d.K, d.dtype, d.group, d.lda, d.ld_codes, d.ld_scales, d.ldr, d.ldo, d.slot = 2, 24, 128, nm.BF16, 64, 128, 64, 2, 24, 24, nm.SLOT_GELU
    for name in ("A", "codes", "scales", "bias", "residual", "out"):
        setattr(d, name, A)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


INVALID, SHAPE, ALIGN, NO_TABLE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5, 8


@pytest.mark.parametrize("change,status", [
    ({"B": -1}, SHAPE), ({"page_size": 0}, SHAPE), ({"max_pages": -1}, SHAPE), ({"max_tokens": -1}, SHAPE), ({"free_capacity": -1}, SHAPE),
    ({"ld_tables": 3}, SHAPE), ({"max_pages": 1 << 20, "page_size": 1 << 12, "ld_tables": 1 << 20}, SHAPE), ({"lengths": None}, INVALID),
    ({"new_tokens": None}, INVALID), ({"free_count": None}, INVALID), ({"block_tables": None}, INVALID), ({"free_pages": None}, INVALID),
    ({"lengths_out": None}, INVALID), ({"free_count_out": None}, INVALID), ({"token_start": None}, INVALID), ({"slots": None}, INVALID),
    ({"positions": None}, INVALID), ({"slots": A + 2}, ALIGN), ({"lengths": A + 1}, ALIGN)])
def test_plan_refusals(lib, ctx, change, status):
    assert lib.nm_kv_plan(ctx, C.byref(plan_desc(**change)), None) == status


@pytest.mark.parametrize("change,status", [
    ({"T": -1}, SHAPE), ({"heads": -1}, SHAPE), ({"kv_heads": -2}, SHAPE), ({"kv_heads": 2 ** 31 - 1}, SHAPE), ({"d": 4}, SHAPE), ({"d": 60}, SHAPE),
    ({"d": 264}, SHAPE), ({"dtype": nm.I8}, UNSUPPORTED), ({"dtype": 9}, UNSUPPORTED), ({"rot": 24}, SHAPE), ({"rot": 72}, SHAPE), ({"rot": -16}, SHAPE),
    ({"rot": 12, "pairs": 1}, SHAPE), ({"rsqrt_slot": 16}, INVALID), ({"rsqrt_slot": -1}, INVALID), ({"rsqrt_slot": 9}, NO_TABLE), ({"qkv": None}, INVALID),
    ({"q_out": None}, INVALID), ({"ld_qkv": 504}, SHAPE), ({"ld_q": 248}, SHAPE), ({"ld_k": 120}, SHAPE), ({"k_cache": None}, INVALID),
    ({"v_cache": None}, INVALID), ({"slots": None}, INVALID), ({"positions": None}, INVALID), ({"cos_sin": None}, INVALID), ({"max_position": 0}, SHAPE),
    ({"num_pages": 0}, SHAPE), ({"page_size": 0}, SHAPE), ({"num_pages": 1 << 16, "page_size": 1 << 16}, SHAPE), ({"stride_token": -64}, SHAPE),
    ({"stride_page": 2044}, ALIGN), ({"stride_head": 68}, ALIGN), ({"qkv": A + 8}, ALIGN), ({"cos_sin": A + 4}, ALIGN), ({"gamma_q": A + 4}, ALIGN),
    ({"slots": A + 1}, ALIGN), ({"ld_qkv": 516}, ALIGN), ({"ld_q": 260}, ALIGN), ({"ld_k": 132}, ALIGN), ({"v_cache": A + 2}, ALIGN)])
def test_rope_refusals(lib, ctx, change, status):
    assert lib.nm_qk_norm_rope_pwl(ctx, C.byref(rope_desc(**change)), None) == status


def test_rope_without_norm_needs_no_table(lib, ctx):
    assert lib.nm_qk_norm_rope_pwl(ctx, C.byref(rope_desc(gamma_q=None, gamma_k=None, rsqrt_slot=9, qkv=None)), None) == INVALID
    assert lib.nm_qk_norm_rope_pwl(ctx, C.byref(rope_desc(T=0, qkv=None)), None) == 0


@pytest.mark.parametrize("change,status", [
    ({"B": -1}, SHAPE), ({"heads": 0}, SHAPE), ({"kv_heads": 0}, SHAPE), ({"kv_heads": 3}, SHAPE), ({"d": 0}, SHAPE), ({"d": 68}, SHAPE), ({"d": 512}, SHAPE),
    ({"dtype": nm.I8}, UNSUPPORTED), ({"max_len": -1}, SHAPE), ({"max_len": 65}, SHAPE), ({"max_pages": -1}, SHAPE), ({"page_size": 0}, SHAPE),
    ({"num_pages": 0}, SHAPE), ({"stride_page": -8}, SHAPE), ({"stride_token": 132}, ALIGN), ({"exp_slot": 7}, NO_TABLE), ({"recip_slot": 99}, INVALID),
    ({"scale": 0.0}, INVALID), ({"scale": -1.0}, INVALID), ({"scale": float("nan")}, INVALID), ({"scale": float("inf")}, INVALID), ({"Q": None}, INVALID),
    ({"k_cache": None}, INVALID), ({"v_cache": None}, INVALID), ({"block_tables": None}, INVALID), ({"lengths": None}, INVALID), ({"out": None}, INVALID),
    ({"ld_q": 504}, SHAPE), ({"ld_out": 504}, SHAPE), ({"ld_tables": 3}, SHAPE), ({"Q": A + 4}, ALIGN), ({"out": A + 8}, ALIGN), ({"ld_q": 516}, ALIGN),
    ({"lengths": A + 2}, ALIGN)])
def test_attention_refusals(lib, ctx, change, status):
    d = attn_desc(**change)
    assert lib.nm_attention_pwl_paged(ctx, C.byref(d), A, 1 << 30, None) == status
    if status in (SHAPE, UNSUPPORTED) and not set(change) & {"ld_q", "ld_out", "ld_tables"}:
        assert lib.nm_attention_paged_workspace_bytes(C.byref(d)) == 0


def test_attention_workspace_refusals(lib, ctx):
    d = attn_desc()
    need = lib.nm_attention_paged_workspace_bytes(C.byref(d))
    if need > 0:
        assert lib.nm_attention_pwl_paged(ctx, C.byref(d), A, need - 1, None) == WORKSPACE
        assert lib.nm_attention_pwl_paged(ctx, C.byref(d), None, need, None) == WORKSPACE
        assert lib.nm_attention_pwl_paged(ctx, C.byref(d), A + 128, need, None) == ALIGN
    assert lib.nm_attention_pwl_paged(ctx, C.byref(attn_desc(B=0, Q=None)), None, 0, None) == 0


@pytest.mark.parametrize("change,status", [
    ({"M": -1}, SHAPE), ({"N": -1}, SHAPE), ({"K": -1}, SHAPE), ({"K": 2 ** 31}, SHAPE), ({"dtype": nm.I8}, UNSUPPORTED), ({"group": 16}, UNSUPPORTED),
    ({"group": 256}, UNSUPPORTED), ({"slot": 16}, INVALID), ({"slot": 8}, NO_TABLE), ({"K": 0}, SHAPE), ({"K": 96}, SHAPE), ({"A": None}, INVALID),
    ({"codes": None}, INVALID), ({"scales": None}, INVALID), ({"out": None}, INVALID), ({"lda": 120}, SHAPE), ({"ld_codes": 48}, SHAPE),
    ({"ld_scales": 1}, SHAPE), ({"ldo": 16}, SHAPE), ({"ldr": 16}, SHAPE), ({"A": A + 8}, ALIGN), ({"codes": A + 8}, ALIGN), ({"scales": A + 1}, ALIGN),
    ({"bias": A + 2}, ALIGN), ({"out": A + 2}, ALIGN), ({"residual": A + 2}, ALIGN), ({"lda": 132}, ALIGN), ({"ld_codes": 72}, ALIGN), ({"ldo": 28}, ALIGN),
    ({"ldr": 28}, ALIGN)])
def test_w4_refusals(lib, ctx, change, status):
    assert lib.nm_linear_pwl_w4(ctx, C.byref(w4_desc(**change)), None) == status


def test_w4_of_nothing(lib, ctx):
    assert lib.nm_linear_pwl_w4(ctx, C.byref(w4_desc(M=0, A=None)), None) == 0
    assert lib.nm_linear_pwl_w4(ctx, C.byref(w4_desc(N=0, codes=None)), None) == 0


def test_counts_that_32_bit_steps_would_pass(lib, ctx):
    big = (1 << 30) + 1
    for name in ("B", "max_tokens", "free_capacity"):
        assert lib.nm_kv_plan(ctx, C.byref(plan_desc(**{name: big})), None) == SHAPE
    assert lib.nm_qk_norm_rope_pwl(ctx, C.byref(rope_desc(T=big)), None) == SHAPE
    long = {"max_pages": 1 << 17, "page_size": 1 << 13, "ld_tables": 1 << 17}
    for change in ({"B": big}, dict(long, max_pages=(1 << 17) + 1, ld_tables=(1 << 17) + 1, max_len=big),
                   dict(long, max_len=1 << 30, B=1 << 18), {"heads": 1 << 25, "ld_q": 1 << 31, "ld_out": 1 << 31}):
        d = attn_desc(**change)
        assert lib.nm_attention_pwl_paged(ctx, C.byref(d), A, 1 << 62, None) == SHAPE
        assert lib.nm_attention_paged_workspace_bytes(C.byref(d)) == 0
    d = attn_desc(**dict(long, max_len=1 << 30, num_pages=1))            # the longest: scores of 2 x 8 rows and some more
    assert 64 << 30 < lib.nm_attention_paged_workspace_bytes(C.byref(d)) < 65 << 30
    for name in ("M", "N", "K"):
        assert lib.nm_linear_pwl_w4(ctx, C.byref(w4_desc(**{name: 1 << 30 | 128})), None) == SHAPE


def test_null_contexts_and_descriptors(lib, ctx):
    assert lib.nm_kv_plan(None, C.byref(plan_desc()), None) == INVALID and lib.nm_kv_plan(ctx, None, None) == INVALID
    assert lib.nm_qk_norm_rope_pwl(None, C.byref(rope_desc()), None) == INVALID and lib.nm_qk_norm_rope_pwl(ctx, None, None) == INVALID
    assert lib.nm_attention_pwl_paged(None, C.byref(attn_desc()), None, 0, None) == INVALID
    assert lib.nm_attention_pwl_paged(ctx, None, None, 0, None) == INVALID and lib.nm_attention_paged_workspace_bytes(None) == 0
    assert lib.nm_linear_pwl_w4(None, C.byref(w4_desc()), None) == INVALID and lib.nm_linear_pwl_w4(ctx, None, None) == INVALID


# ---------------------------------------------------------------- the binding


def z(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_binding_refuses_wrong_types_shapes_and_strides(lib):
    i, c = torch.int32, nm.Context
    table, lens = z(2, 4, dtype=i), z(2, dtype=i)
    q, cache = z(2, 8, 64), z(9, 16, 2, 64)
    good = dict(q=q, k_cache=cache, v_cache=cache, block_tables=table, lengths=lens, out=torch.empty_like(q))
    if not torch.cuda.is_available():
        c.attn_paged_desc(**good)
    for bad in ({"lengths": lens.long()}, {"block_tables": table.long()}, {"lengths": z(3, dtype=i)}, {"out": q.float()}, {"out": z(2, 8, 128)[..., ::2]},
                {"q": z(2, 64, 8).transpose(1, 2)}, {"k_cache": z(9, 16, 2, 128)}, {"v_cache": z(9, 2, 16, 64).transpose(1, 2)}, {"k_cache": cache.half()},
                {"block_tables": z(4, 2, dtype=i).t()}, {"q": z(2, 16, 64)[:, ::2]}, {"k_cache": z(9, 16, 64)}):
        with pytest.raises(ValueError):
            c.attn_paged_desc(**dict(good, **bad))
    a, codes, scales, out = z(3, 128), z(24, 64, dtype=torch.uint8), z(24, 2), z(3, 24)
    for bad in ((a, codes.to(torch.int8), scales, out), (a, codes, scales.float(), out), (a, codes, z(24, 3), out), (a, codes, scales, z(3, 25)),
                (a, z(24, 63, dtype=torch.uint8), scales, out), (a.t().contiguous().t(), codes, scales, out), (a, codes, z(24, 0), out)):
        with pytest.raises(ValueError):
            c.linear_w4_desc(*bad)
    qkv, qo = z(3, 512), z(3, 256)
    for bad in ({"positions": z(3)}, {"positions": z(2, dtype=i)}, {"positions": None}, {"cos_sin": z(100, 32)}, {"gamma_q": z(64)},
                {"gamma_k": z(32, dtype=torch.float32)}, {"k_cache": cache}, {"k_cache": cache, "v_cache": cache}, {"slots": z(3, dtype=torch.int64)},
                {"k_out": z(3, 64)}, {"cos_sin": z(32, 100, dtype=torch.float32).t()}):
        kw = dict({"positions": z(3, dtype=i), "cos_sin": z(100, 32, dtype=torch.float32)}, **bad)
        with pytest.raises(ValueError):
            c.qk_rope_desc(qkv, 4, 2, 64, qo, **kw)
    arrays = dict(lengths=lens, new_tokens=lens, block_tables=table, free_pages=z(9, dtype=i), free_count=z(1, dtype=i), page_size=16, lengths_out=lens,
                  free_count_out=z(1, dtype=i), token_start=z(3, dtype=i), slots=z(4, dtype=i), positions=z(4, dtype=i))
    for name in arrays:
        if name != "page_size":
            with pytest.raises(ValueError):
                c.kv_plan_desc(**dict(arrays, **{name: arrays[name].long()}))
    for name in ("new_tokens", "lengths_out", "token_start", "positions", "free_count"):
        with pytest.raises(ValueError):
            c.kv_plan_desc(**dict(arrays, **{name: z(7, dtype=i)}))


def test_reference_plan_on_a_worked_example():
    tables = np.array([[4, 5, 0], [6, 0, 0], [7, 8, 9]], np.int32)
    free = np.array([1, 2, 3, 0, 0, 0, 0], np.int32)
    status, out = ref.plan([5, 4, 9], [1, 3, -1], tables, free, 3, 4, 6)
    assert status == 0
    # request 2's pages are pushed (stack 1 2 3 7 8 9), request 1 takes the last one
    assert free.tolist() == [1, 2, 3, 7, 8, 9, 0] and tables[1].tolist() == [6, 9, 0] and out["free_count"] == 5
    assert out["lengths"] == [6, 7, 0] and out["token_start"] == [0, 1, 4, 4]
    assert out["slots"] == [21, 36, 37, 38, -1, -1] and out["positions"] == [5, 4, 5, 6, 0, 0]
