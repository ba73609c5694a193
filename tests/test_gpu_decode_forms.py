"""GPU tests of the decoding operators in the forms and combinations that their neighbours' tests leave out."""
import numpy as np
import pytest
import torch

import decode_ref as ref
from decode_ref import TYPES, check, f64
from test_gpu_decode import cache_views, check_attention, ctx, gen_of, i32, make_cache, randn  # noqa: F401

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
