"""CPU-only checks of the decoding operators' entry points: calls that a launch must never see."""
import ctypes as C

import pytest
import torch

import paper_2305_14405_b200 as nm
from test_decode_host import A, ALIGN, INVALID, NO_TABLE, SHAPE, attn_desc, ctx, lib, rope_desc  # noqa: F401


@pytest.mark.parametrize("slot", [-1, 16, 99, -2 ** 31])
@pytest.mark.parametrize("norm", [{"heads": 0, "gamma_k": None}, {"kv_heads": 0, "gamma_q": None}, {"heads": 0}, {"kv_heads": 0}])
def test_rope_table_of_no_heads(lib, ctx, norm, slot):  # noqa: F811
    """A gamma for heads that are not there needs no table, but a number that is no slot is refused all the same."""
    assert lib.nm_qk_norm_rope_pwl(ctx, C.byref(rope_desc(rsqrt_slot=slot, **norm)), None) == INVALID


def test_rope_table_that_is_not_needed(lib, ctx):  # noqa: F811
    no_launch = 6   # all arguments passed; there is no device
    for norm in ({"heads": 0, "gamma_k": None}, {"kv_heads": 0, "gamma_q": None}):
        assert lib.nm_qk_norm_rope_pwl(ctx, C.byref(rope_desc(rsqrt_slot=9, **norm)), None) == no_launch   # slot 9 holds no table
    assert lib.nm_qk_norm_rope_pwl(ctx, C.byref(rope_desc(rsqrt_slot=9, heads=0)), None) == NO_TABLE
    assert lib.nm_qk_norm_rope_pwl(ctx, C.byref(rope_desc(rsqrt_slot=99, gamma_q=None, gamma_k=None)), None) == no_launch


def test_rows_whose_steps_would_not_fit_32_bits(lib, ctx):  # noqa: F811
    """Threads step through a token's row by some hundreds, and count the heads that fill up its last groups."""
    wide, heads = 1 << 31, 1 << 24   # 2^30 elements of 64 channels and some more
    assert lib.nm_qk_norm_rope_pwl(ctx, C.byref(rope_desc(heads=heads, ld_qkv=wide, ld_q=wide)), None) == SHAPE
    d = attn_desc(heads=heads + 2, ld_q=wide, ld_out=wide)
    assert lib.nm_attention_pwl_paged(ctx, C.byref(d), A, 1 << 40, None) == SHAPE
    assert lib.nm_attention_paged_workspace_bytes(C.byref(d)) == 0


@pytest.mark.parametrize("change,status", [({"rows": -1}, SHAPE), ({"rows": (1 << 30) + 1}, SHAPE), ({"token_start": A + 2}, ALIGN), ({"rows": 0, "Q": None}, 0),
                                           ({"rows": 3, "Q": None}, INVALID), ({"rows": 3, "max_len": 65}, SHAPE)])
def test_attention_with_rows_of_a_plan(lib, ctx, change, status):  # noqa: F811
    d = attn_desc(**dict({"token_start": A, "rows": 5}, **change))
    assert lib.nm_attention_pwl_paged(ctx, C.byref(d), A, 1 << 30, None) == status


def test_binding_of_the_rows_of_a_plan(lib):  # noqa: F811
    if torch.cuda.is_available():
        pytest.skip("a machine without a device")
    i = torch.int32
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)  # noqa: E731
    cache = z(9, 16, 2, 64)
    good = dict(q=z(11, 8, 64), k_cache=cache, v_cache=cache, block_tables=z(2, 4, dtype=i), lengths=z(2, dtype=i), out=z(11, 8, 64), token_start=z(3, dtype=i))
    d = nm.Context.attn_paged_desc(**good)
    assert (d.B, d.rows, d.ld_q, d.ld_out) == (2, 11, 512, 512) and d.token_start
    d = nm.Context.attn_paged_desc(**dict(good, q=z(1, 8, 64), out=z(1, 8, 64)))
    assert (d.B, d.rows, d.ld_q) == (2, 1, 512)
    for bad in ({"token_start": z(2, dtype=i)}, {"token_start": z(12, dtype=i)}, {"token_start": z(3, dtype=torch.int64)}, {"lengths": z(11, dtype=i)},
                {"out": z(2, 8, 64)}, {"block_tables": z(4, dtype=i)}, {"token_start": None}):
        with pytest.raises(ValueError):
            nm.Context.attn_paged_desc(**dict(good, **bad))


# ---------------------------------------------------------------- what only the binding can see


class FakeLibrary:
    """Notes what would have been launched."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append(name) or 0


@pytest.fixture
def binding():
    """A context of device 0 without a device, and the four calls with descriptors of tensors that lie nowhere."""
    if torch.cuda.is_available():
        pytest.skip("a machine without a device")
    c = object.__new__(nm.Context)
    c._lib, c._h, c._raw_stream, c.device = FakeLibrary(), None, lambda device: 0, 0
    i = torch.int32
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)  # noqa: E731
    cache, n = z(9, 16, 2, 64), z(2, dtype=i)
    plan = c.kv_plan_desc(n, n, z(2, 4, dtype=i), z(9, dtype=i), z(1, dtype=i), 16, n, z(1, dtype=i), z(3, dtype=i), z(4, dtype=i), z(4, dtype=i))
    calls = {"kv_plan": plan, "qk_norm_rope_pwl": c.qk_rope_desc(z(3, 512), 4, 2, 64, z(3, 256)),
             "attention_pwl_paged": c.attn_paged_desc(z(2, 8, 64), cache, cache, z(2, 4, dtype=i), n, z(2, 8, 64)),
             "linear_pwl_w4": c.linear_w4_desc(z(3, 128), z(24, 64, dtype=torch.uint8), z(24, 2), z(3, 24))}
    return c, calls


class Fake:
    """As much of a tensor as a check of its place looks at."""

    def __init__(self, device, size=1 << 20, contiguous=True):
        self.device, self._size, self._contiguous = torch.device(device), size, contiguous

    def get_device(self):
        return -1 if self.device.type == "cpu" else self.device.index

    def is_contiguous(self):
        return self._contiguous

    def numel(self):
        return self._size

    def element_size(self):
        return 1

    def data_ptr(self):
        return A


def test_descriptors_of_another_device_are_refused(binding):
    c, calls = binding
    for name, desc in calls.items():
        for device in (1, 7):
            desc.device = device
            with pytest.raises(ValueError):
                getattr(c, name)(desc)
    assert not c._lib.calls
    for name, desc in calls.items():
        desc.device = 0
        getattr(c, name)(desc)
    assert c._lib.calls == ["nm_" + name for name in calls]


def test_descriptors_know_their_device():
    assert nm._same_device([None, Fake("cuda:1"), Fake("cuda:1")]) == 1 and nm._same_device([Fake("cuda:0")]) == 0
    assert nm._same_device([Fake("cpu"), Fake("cpu")]) is None
    with pytest.raises(ValueError):
        nm._same_device([Fake("cuda:1"), Fake("cuda:0")])
    with pytest.raises(ValueError):
        nm._same_device([Fake("cuda:0"), Fake("cpu")])


@pytest.mark.parametrize("workspace", [Fake("cpu"), Fake("cuda:1"), Fake("cuda:0", contiguous=False), torch.zeros(1 << 12, dtype=torch.uint8)])
def test_workspaces_that_the_kernels_must_not_write_are_refused(binding, workspace):
    c, calls = binding
    with pytest.raises(ValueError):
        c.attention_pwl_paged(calls["attention_pwl_paged"], workspace)
    assert not c._lib.calls
    c.attention_pwl_paged(calls["attention_pwl_paged"], Fake("cuda:0"))
    c.attention_pwl_paged(calls["attention_pwl_paged"])
    assert len(c._lib.calls) == 2


def test_strides_of_extents_of_one_do_not_count(lib):  # noqa: F811
    """With one key head (or one page, or pages of one token) the distance of heads is never used: K and V may differ in it."""
    if torch.cuda.is_available():
        pytest.skip("a machine without a device")
    i = torch.int32
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)  # noqa: E731
    k, v = z(9, 16, 1, 64), z(9, 1, 16, 64).transpose(1, 2)   # the same places, other strides of the one head
    d = nm.Context.attn_paged_desc(z(2, 8, 64), k, v, z(2, 4, dtype=i), z(2, dtype=i), z(2, 8, 64))
    assert (d.stride_page, d.stride_token, d.stride_head) == (1024, 64, 0)
    d = nm.Context.qk_rope_desc(z(3, 384), 4, 1, 64, z(3, 256), k_cache=v, v_cache=k, slots=z(3, dtype=i))
    assert (d.stride_page, d.stride_token, d.stride_head) == (1024, 64, 0)
    with pytest.raises(ValueError):   # two heads: their distance counts
        nm.Context.attn_paged_desc(z(2, 8, 64), z(9, 16, 2, 64), z(9, 2, 16, 64).transpose(1, 2), z(2, 4, dtype=i), z(2, dtype=i), z(2, 8, 64))


def test_numbers_that_do_not_fit_a_descriptor_are_refused(lib):  # noqa: F811
    """32-bit fields would silently take a number's lower bits: pages of 2^32 + 16 tokens are no pages of 16."""
    if torch.cuda.is_available():
        pytest.skip("a machine without a device")
    i, c = torch.int32, nm.Context
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)  # noqa: E731
    n, cache = z(2, dtype=i), z(9, 16, 2, 64)
    with pytest.raises(ValueError):
        c.kv_plan_desc(n, n, z(2, 4, dtype=i), z(9, dtype=i), z(1, dtype=i), 2 ** 32 + 16, n, z(1, dtype=i), z(3, dtype=i), z(4, dtype=i), z(4, dtype=i))
    good = (z(2, 8, 64), cache, cache, z(2, 4, dtype=i), n, z(2, 8, 64))
    for bad in ({"max_len": 2 ** 32 + 8}, {"max_len": 2 ** 31}, {"max_len": -2 ** 31 - 1}, {"exp_slot": 2 ** 32 + nm.SLOT_EXP}, {"recip_slot": -2 ** 32}):
        with pytest.raises(ValueError):
            c.attn_paged_desc(*good, **bad)
    long = torch.empty((1, 1 << 20), dtype=i)   # a table of 2^20 pages of 4096 tokens: 2^32
    with pytest.raises(ValueError):
        c.attn_paged_desc(z(1, 1, 8), z(1, 4096, 1, 8), z(1, 4096, 1, 8), long, n[:1], z(1, 1, 8))
    d = c.attn_paged_desc(z(1, 1, 8), z(1, 4096, 1, 8), z(1, 4096, 1, 8), long, n[:1], z(1, 1, 8), max_len=4096)
    assert d.max_len == 4096 and d.max_pages == 1 << 20
    with pytest.raises(ValueError):
        c.linear_w4_desc(z(3, 128), z(24, 64, dtype=torch.uint8), z(24, 2), z(3, 24), slot=2 ** 32)
