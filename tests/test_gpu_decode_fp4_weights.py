"""Weights of decode attention over caches held in 4 bits, bf16: good to 2^-16 of themselves.

48 rows whose key is 1 in one dim and whose value is 0, and one whose key is 0 and whose value is 1: against a query that is x in that dim and 0 elsewhere,
every sum of products is exact, the weights are 1 and w = e^-x, and the result is w / (48 + w).  What it may be off by, relative, u = 2^-24: the weight's own 2^-16; its exponent,
x log2(e) below 2, 2 u for the constant and the scale, 3 u for the reference and the difference from it, times ln 2; exp2 of the hardware 2 u; sums over the
pieces and the division, 4 u.  16 u are more than these together."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2605_23258_amd import binding as vb
from paper_2605_23258_amd import datagen as dg
from paper_2605_23258_amd import pipeline as pl
from test_gpu_decode_fp4 import dev

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("d,G", [(128, 1), (128, 4), (128, 7), (128, 16), (64, 2), (64, 8), (64, 12)])
def test_weights_to_2_16(d, G):
    B, H, n = 56, 4, 48
    rng = np.random.default_rng(d + G)
    q = np.zeros((B, H * G, d), dtype=np.float32)
    q[:, :, 5] = rng.uniform(0.05, 1.38, (B, H * G))
    bits = dg.f32_to_bf16_bits(q)
    x = dg.widen(bits)[:, :, 5]
    codes, ones = np.zeros((B, H, n + 1, d // 2), dtype=np.uint8), np.zeros((B, H, n + 1, d // 2), dtype=np.uint8)
    codes[:, :, :n, 2] = 2 << 4                        # element 5: 1
    ones[:, :, n] = 2 | 2 << 4
    k, v, scales = dev(codes), dev(ones), torch.full((B, H, n + 1, d // 32), 127, dtype=torch.uint8, device=DEV)
    live, q_dev, out = torch.full((B,), n + 1, dtype=torch.int32, device=DEV), dev(bits.view(np.int16)).view(torch.bfloat16), torch.empty(B, H * G, d, device=DEV)
    c = vb.CacheFp4(batch=B, n_q_heads=H * G, n_kv_heads=H, head_dim=d, dtype=vb.VECTOR_BF16, cap_retain=n + 1, n_approx=0)
    c.len_retain, c.k_ret, c.k_ret_scale, c.v_ret, c.v_ret_scale = live.data_ptr(), k.data_ptr(), scales.data_ptr(), v.data_ptr(), scales.data_ptr()
    vb.vector_decode_attn_fp4(c, q_dev, 1.0, out, pl.alloc_workspace(vb.vector_decode_fp4_workspace_bytes(c)), flags=vb.VECTOR_DECODE_OUT_F32)
    got, want = out.double().cpu().numpy(), np.exp(-x) / (n + np.exp(-x))
    off = np.abs(got / want[:, :, None] - 1)
    assert off.max() <= 2.0 ** -16 + 16 * 2.0 ** -24, f"{(off.max(axis=2) > 2.0 ** -16 + 16 * 2.0 ** -24).sum()} of {x.size} weights, {off.max() * 2 ** 16:.3f} of 2^-16"
