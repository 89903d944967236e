"""The FP4 form of the experts (E2M1 elements, a power of two per 32 of K) against its oracle, through the C ABI."""
import numpy as np
import pytest
import torch

from oracle import fp4_oracle as Q
from oracle import moe_oracle as O
from paper_2605_05607_b200 import binding as B
from tests import helpers as H

pytestmark = pytest.mark.gpu


def f64(t):
    return O.bf16_to_f64(H.bf16_host(t))


def rows_fp4(x):
    R, K = x.shape
    q = torch.full((R, K // 2), 0xA5, dtype=torch.uint8, device="cuda")
    s = torch.full((R, K // 32), 0xA5, dtype=torch.uint8, device="cuda")
    B.moe_quantize_rows_fp4(x, q, s)
    return q, s


def weights_fp4(w):
    E, K, N = w.shape
    q = torch.full((E, N, K // 2), 0xA5, dtype=torch.uint8, device="cuda")
    s = torch.full((B.moe_fp4_scale_bytes(E, K, N),), 0xA5, dtype=torch.uint8, device="cuda")
    B.moe_quantize_weights_fp4(w, q, s)
    return q, s


@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 64), (7, 96), (300, 2880), (513, 4096), (5000, 1536)])
def test_quantize_rows_bit_exact(rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x = (x * torch.exp2(torch.randint(-30, 30, (rows, cols // 32, 1), generator=g, device="cuda").float()).expand(-1, -1, 32).reshape(rows, cols)).bfloat16()
    q, s = rows_fp4(x)
    q_ref, s_ref = Q.quantize_rows(f64(x))
    assert np.array_equal(s.cpu().numpy(), s_ref)
    assert np.array_equal(q.cpu().numpy(), q_ref)
    back = torch.full_like(x, 7.0)
    B.moe_dequantize_rows_fp4(q, s, back)
    assert np.array_equal(f64(back), Q.dequantize_rows(q_ref, s_ref))


def test_quantize_rows_every_border_and_extreme():
    """Every value of the grid, every midpoint and its neighbours in bf16, at the exponents where something changes; blocks of zeros, of
    subnormals, of the largest value, and blocks that hold an infinity or a NaN."""
    mags = np.concatenate([Q.GRID, Q.BORDER, Q.BORDER * (1 + 2.0 ** -7), Q.BORDER * (1 - 2.0 ** -8)])
    mags = np.concatenate([mags, -mags])
    blocks = []
    for ex in (-140, -131, -128, -127, -126, -125, -60, 0, 1, 60, 120, 124, 125):
        for top in (4.0, 4.5, 6.0, 7.0, 7.96875):
            for part in np.array_split(mags, 2):
                b = np.zeros(32)
                b[:part.size] = part[:31]
                b[31] = top
                with np.errstate(over="ignore"):
                    blocks.append(np.ldexp(b, ex))
    blocks.append(np.zeros(32))
    blocks.append(-np.zeros(32))
    blocks.append(np.full(32, 2.0 ** -133))
    x = torch.tensor(np.stack(blocks), dtype=torch.float64).to(torch.bfloat16).cuda()
    finite = torch.isfinite(x).all(1).cpu().numpy()
    q, s = rows_fp4(x)
    q_ref, s_ref = Q.quantize_rows(f64(x)[finite])
    assert np.array_equal(s.cpu().numpy()[finite], s_ref)
    assert np.array_equal(q.cpu().numpy()[finite], q_ref)
    back = torch.zeros_like(x)
    B.moe_dequantize_rows_fp4(q, s, back)
    assert np.array_equal(f64(back)[finite], Q.dequantize_rows(q_ref, s_ref))
    bad = torch.ones(4, 64, device="cuda").bfloat16()
    bad[0, 3], bad[1, 40], bad[2, 63] = float("nan"), float("inf"), -float("inf")
    q, s = rows_fp4(bad)
    assert s.cpu().tolist() == [[255, 125], [125, 255], [125, 255], [125, 125]]
    back = torch.zeros_like(bad)
    B.moe_dequantize_rows_fp4(q, s, back)
    nan = torch.isnan(back).view(4, 2, 32)
    assert torch.equal(nan.all(-1), (s == 255)) and torch.equal(nan.any(-1), (s == 255))
    assert (back.view(4, 2, 32)[~nan.any(-1)] == 1).all()


def test_dequantize_rows_every_code_at_every_scale():
    codes = torch.arange(16, dtype=torch.uint8).repeat(2).repeat(255, 1)
    packed = (codes[:, 0::2] | (codes[:, 1::2] << 4)).cuda()
    scale = torch.arange(255, dtype=torch.uint8).view(-1, 1).cuda()
    back = torch.zeros(255, 32, device="cuda").bfloat16()
    B.moe_dequantize_rows_fp4(packed, scale, back)
    want = torch.tensor(Q.dequantize_rows(packed.cpu().numpy(), scale.cpu().numpy())).to(torch.bfloat16)   # infinite at the very top
    assert torch.equal(back.cpu(), want)


def test_fp4_of_no_rows():
    e = torch.empty(0, 64, device="cuda").bfloat16()
    u = torch.empty(0, 32, dtype=torch.uint8, device="cuda")
    B.moe_quantize_rows_fp4(e, u, u)
    B.moe_dequantize_rows_fp4(u, u, e)


@pytest.mark.parametrize("E,K,N", [(1, 32, 8), (3, 96, 40), (2, 256, 128), (2, 288, 136), (1, 2880, 264), (5, 544, 72), (2, 768, 2880)])
def test_quantize_weights_bit_exact(E, K, N):
    g = torch.Generator(device="cuda").manual_seed(K + N)
    w = (torch.randn(E, K, N, generator=g, device="cuda") * torch.exp2(torch.randint(-9, 9, (E, 1, N), generator=g, device="cuda").float())).bfloat16()
    w[0, :32, 1] = 0
    q, s = weights_fp4(w)
    q_ref, s_ref = Q.quantize_weights(f64(w))
    assert np.array_equal(q.cpu().numpy(), q_ref)
    assert s.numel() == Q.scale_bytes(E, K, N)
    assert np.array_equal(s.cpu().numpy(), Q.tile_scales(s_ref))
    back = torch.full_like(w, 7.0)
    B.moe_dequantize_weights_fp4(q, s, back)
    want = np.stack([Q.dequantize_rows(q_ref[e], s_ref[e]).T for e in range(E)])
    assert np.array_equal(f64(back), want)
