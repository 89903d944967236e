"""Refusals of the norm and the 4-bit operators, which come before any device is touched, and pins of their oracles."""
import ctypes
import re

import numpy as np
import pytest
import torch

from oracle import fp4_oracle as Q
from oracle import norm_oracle as N
from paper_2605_05607_b200 import binding as B
from paper_2605_05607_b200 import build

OK, ARG, SHAPE, SMALL, ALIGN, CUDA = (B.MOE_OK, B.MOE_ERR_INVALID_ARG, B.MOE_ERR_UNSUPPORTED_SHAPE, B.MOE_ERR_WORKSPACE_TOO_SMALL,
                                      B.MOE_ERR_MISALIGNED, B.MOE_ERR_CUDA)
P = 1 << 20                      # an address that is never read: every call here is refused, or finds no device
NO_GPU = not torch.cuda.is_available()


@pytest.fixture(scope="module")
def L():
    build.build_library()
    return B.lib()


@pytest.mark.parametrize("change,code", [
    (dict(rows=-1), ARG), (dict(cols=0), ARG), (dict(weight=None), ARG), (dict(x=None), ARG), (dict(y=None, yq=None, scale=None), ARG),
    (dict(yq=None), ARG), (dict(scale=None), ARG), (dict(residual=None), ARG), (dict(res_out=P), ARG), (dict(eps=-1.0), ARG),
    (dict(eps=float("nan")), ARG), (dict(eps=float("inf")), ARG), (dict(cols=100), SHAPE), (dict(cols=16392), SHAPE), (dict(rows=1 << 40), SHAPE),
    (dict(x=P + 2), ALIGN), (dict(weight=P + 4), ALIGN), (dict(residual=P + 8), ALIGN), (dict(y=P + 8), ALIGN), (dict(yq=P + 4), ALIGN),
    (dict(scale=P + 2), ALIGN), (dict(rstd=P + 1), ALIGN), (dict(res_out=P + 8), ALIGN),
], ids=str)
def test_rmsnorm_refuses(L, change, code):
    a = dict(x=P, residual=P, weight=P, w32=0, eps=1e-6, rows=4, cols=64, res_out=2 * P, y=P, yq=P, scale=P, rstd=P) | change
    assert L.moe_rmsnorm(*a.values(), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(dy=None), ARG), (dict(s=None), ARG), (dict(weight=None), ARG), (dict(rstd=None), ARG), (dict(dx=None), ARG), (dict(dw=None), ARG),
    (dict(ws=None), ARG), (dict(rows=-1), ARG), (dict(cols=12), SHAPE), (dict(cols=16392), SHAPE), (dict(rows=1 << 31), SHAPE),
    (dict(ws_bytes=1023), SMALL), (dict(dy=P + 8), ALIGN), (dict(dres=P + 8), ALIGN), (dict(dw=P + 4), ALIGN), (dict(ws=P + 8), ALIGN),
    (dict(rstd=P + 2), ALIGN),
], ids=str)
def test_rmsnorm_backward_refuses(L, change, code):
    a = dict(dy=P, dres=None, s=P, weight=P, w32=1, rstd=P, rows=4, cols=64, dx=P, dw=P, ws=P, ws_bytes=1024) | change
    assert L.moe_rmsnorm_backward(*a.values(), None) == code


def test_rmsnorm_backward_workspace(L):
    assert B.moe_rmsnorm_backward_workspace_bytes(0, 64) == 0
    assert B.moe_rmsnorm_backward_workspace_bytes(4, 64) == 1024
    most = B.moe_rmsnorm_backward_workspace_bytes(1 << 20, 4096)
    assert most == B.moe_rmsnorm_backward_workspace_bytes(1 << 30, 4096) <= 16 << 20
    out = ctypes.c_size_t(0)
    assert L.moe_rmsnorm_backward_workspace_bytes(4, 60, ctypes.byref(out)) == SHAPE
    assert L.moe_rmsnorm_backward_workspace_bytes(4, 64, None) == ARG


@pytest.mark.parametrize("fn,change,code", [
    (fn, c, code) for fn in ("moe_quantize_rows_fp4", "moe_dequantize_rows_fp4") for c, code in (
        (dict(src=None), ARG), (dict(rows=-1), ARG), (dict(cols=0), ARG), (dict(dst=None), ARG), (dict(cols=48), SHAPE), (dict(rows=1 << 32), SHAPE),
        (dict(src=P + 2), ALIGN), (dict(dst=P + 2), ALIGN))
] + [("moe_quantize_rows_fp4", dict(scale=None), ARG)], ids=str)
def test_rows_fp4_refuse(L, fn, change, code):
    a = dict(src=P, rows=4, cols=64, dst=P, scale=P) | change
    order = ("src", "rows", "cols", "dst", "scale") if fn == "moe_quantize_rows_fp4" else ("src", "scale", "rows", "cols", "dst")
    assert getattr(L, fn)(*[a[n] for n in order], None) == code


@pytest.mark.parametrize("fn,change,code", [
    (fn, c, code) for fn in ("moe_quantize_weights_fp4", "moe_dequantize_weights_fp4") for c, code in (
        (dict(w=None), ARG), (dict(wq=None), ARG), (dict(scale=None), ARG), (dict(E=0), ARG), (dict(E=70000), ARG), (dict(K=-32), ARG), (dict(N=0), ARG),
        (dict(K=40), SHAPE), (dict(N=12), SHAPE), (dict(w=P + 8), ALIGN), (dict(wq=P + 4), ALIGN), (dict(scale=P + 8), ALIGN))
], ids=str)
def test_weights_fp4_refuse(L, fn, change, code):
    a = dict(w=P, wq=P, scale=P, E=2, K=64, N=64) | change
    order = ("w", "E", "K", "N", "wq", "scale") if fn == "moe_quantize_weights_fp4" else ("wq", "scale", "E", "K", "N", "w")
    assert getattr(L, fn)(*[a[n] for n in order], None) == code


def test_fp4_scale_bytes(L):
    assert B.moe_fp4_scale_bytes(1, 32, 8) == 1024
    for E, K, N in ((3, 4096, 1536), (2, 288, 136), (5, 2880, 2880)):
        assert B.moe_fp4_scale_bytes(E, K, N) == Q.scale_bytes(E, K, N)
    out = ctypes.c_size_t(0)
    assert L.moe_fp4_scale_bytes(0, 32, 8, ctypes.byref(out)) == ARG and L.moe_fp4_scale_bytes(1, 32, 8, None) == ARG


def shape(**kw):
    a = dict(T=16, d=64, f=96, E=4, k=2, G=2, score_fn=0, flags=0) | kw
    return B.MoEShape(*a.values())


def layout(ptr=P):
    return B.MoELayoutC(*[ptr] * 9)


BAD_FLAGS = [B.MOE_FLAG_FUSED_FFN, B.MOE_FLAG_COMBINE_IN_EPILOGUE, B.MOE_FLAG_GEMM1_PAIR, B.MOE_FLAG_GEMM1_GATHER, B.MOE_FLAG_GEMM2_PAIR,
             B.MOE_FLAG_GEMM2_SINGLE, B.MOE_FLAG_FUSED_FFN | B.MOE_FLAG_TRACK_DISPATCH]


@pytest.mark.parametrize("kw,change,code", [
    (dict(d=48), {}, SHAPE), (dict(f=80), {}, SHAPE), (dict(E=3), {}, ARG), *[(dict(flags=f), {}, ARG) for f in BAD_FLAGS],
    *[({}, {n: None}, ARG) for n in ("xq", "sx", "w", "w1", "s1", "w3", "s3", "w2", "s2", "o", "ws")],
    *[({}, {n: P + 64}, ALIGN) for n in ("xq", "w1", "w3", "w2", "o", "ws")], *[({}, {n: P + 8}, ALIGN) for n in ("w", "s1", "s3", "s2")],
    ({}, dict(bytes=1000), SMALL),
], ids=str)
def test_expert_ffn_fp4_refuses(L, kw, change, code):
    a = dict(xq=P, sx=P, lay=ctypes.byref(layout()), w=P, w1=P, s1=P, w3=P, s3=P, w2=P, s2=P, o=P, ws=P, bytes=1 << 30) | change
    assert L.moe_expert_ffn_fp4(ctypes.byref(shape(**kw)), *a.values(), None) == code


def test_expert_ffn_fp4_refuses_layouts(L):
    args = (P, P, P, P, P, P, P, P, P, P, 1 << 30, None)
    assert L.moe_expert_ffn_fp4(ctypes.byref(shape()), P, P, None, *args[1:]) == ARG
    assert L.moe_expert_ffn_fp4(ctypes.byref(shape()), P, P, ctypes.byref(layout(P + 4)), *args[1:]) == ALIGN
    assert L.moe_expert_ffn_fp4(None, P, P, ctypes.byref(layout()), *args[1:]) == ARG


@pytest.mark.parametrize("kw,change,code", [
    (dict(d=48), {}, SHAPE), (dict(f=80), {}, SHAPE), *[(dict(flags=f), {}, ARG) for f in BAD_FLAGS], (dict(flags=B.MOE_FLAG_SPARSE_TOPK), {}, ARG),
    *[({}, {n: None}, ARG) for n in ("x", "wg", "w1", "s1", "w3", "s3", "w2", "s2", "y", "ws")],
    *[({}, {n: P + 64}, ALIGN) for n in ("x", "w1", "w3", "w2", "y", "ws")], *[({}, {n: P + 8}, ALIGN) for n in ("wg", "s1", "s3", "s2", "logits")],
    ({}, dict(bytes=1000), SMALL), ({}, dict(bias=P, stride=3), ARG),
], ids=str)
def test_layer_fp4_refuses(L, kw, change, code):
    a = dict(x=P, wg=P, bias=None, stride=0, w1=P, s1=P, w3=P, s3=P, w2=P, s2=P, y=P, logits=None, idx=None, w=None, lay=None, ws=P, bytes=1 << 30) | change
    assert L.moe_layer_fp4(ctypes.byref(shape(**kw)), *a.values(), None) == code


@pytest.mark.skipif(not NO_GPU, reason="what is said without a device")
def test_no_device_is_an_error(L):
    lay = ctypes.byref(layout())
    assert L.moe_rmsnorm(P, None, P, 0, 1e-6, 4, 64, None, P, None, None, None, None) == CUDA
    assert L.moe_rmsnorm_backward(P, None, P, P, 0, P, 4, 64, P, P, P, 1024, None) == CUDA
    assert L.moe_quantize_rows_fp4(P, 4, 64, P, P, None) == CUDA
    assert L.moe_dequantize_rows_fp4(P, P, 4, 64, P, None) == CUDA
    assert L.moe_quantize_weights_fp4(P, 1, 64, 64, P, P, None) == CUDA
    assert L.moe_dequantize_weights_fp4(P, P, 1, 64, 64, P, None) == CUDA
    assert L.moe_expert_ffn_fp4(ctypes.byref(shape()), P, P, lay, P, P, P, P, P, P, P, P, P, 1 << 30, None) == CUDA
    assert L.moe_layer_fp4(ctypes.byref(shape()), P, P, None, 0, P, P, P, P, P, P, P, None, None, None, None, P, 1 << 30, None) == CUDA


# ---- the oracles ------------------------------------------------------------------------------------------------------------
def test_fp4_codes_against_search():
    """Nearest element by search over all sixteen, ties to the even code; the block's exponent from its largest value."""
    rng = np.random.default_rng(1)
    v = np.concatenate([rng.standard_normal((200, 32)) * np.exp2(rng.integers(-20, 20, (200, 1))), np.tile(Q.BORDER, (1, 5))[:, :32]])
    ex = Q.exponents(v)[:, 0]
    codes = Q.codes_of(v, Q.exponents(v))
    for row, e, c in zip(v, ex, codes):
        assert 4 <= np.abs(row).max() / 2.0 ** e < 8
        for x, got in zip(row / 2.0 ** e, c):
            x = np.clip(x, -6, 6)
            dist = np.abs(Q.GRID - abs(x))
            best = np.flatnonzero(dist == dist.min())
            want = best[best % 2 == 0][0] if best.size > 1 else best[0]
            assert (got & 7) == want and bool(got & 8) == bool(np.signbit(x))


def test_fp4_exact_values_survive_and_scales_have_their_places():
    grid = np.concatenate([Q.GRID, -Q.GRID, Q.GRID, Q.GRID])[None, :] * 2.0 ** np.array([[-9], [0], [7]])
    packed, scale = Q.quantize_rows(grid)
    assert np.array_equal(Q.dequantize_rows(packed, scale), grid) and scale[:, 0].tolist() == [118, 127, 134]
    s = np.arange(2 * 136 * 9, dtype=np.int64).reshape(2, 136, 9) % 251
    tiles = Q.tile_scales(s.astype(np.uint8))
    assert tiles.size == 2 * 2 * 2 * 1024
    assert tiles[0] == s[0, 0, 0] and tiles[1] == s[0, 0, 1] and tiles[4] == s[0, 32, 0] and tiles[16] == s[0, 1, 0]
    assert tiles[512] == s[0, 0, 4] and tiles[1024] == s[0, 0, 8] and tiles[1025] == 127 and tiles[2048] == s[0, 128, 0]
    assert tiles[4096] == s[1, 0, 0]
    assert Q.quantize_rows(np.zeros((1, 32)))[1][0, 0] == 127 and Q.quantize_rows(np.full((1, 32), 2.0 ** -133))[1][0, 0] == 0


def test_norm_oracle_against_differences():
    rng = np.random.default_rng(2)
    x, r, w, c = rng.standard_normal((3, 24)), rng.standard_normal((3, 24)), rng.standard_normal(24), rng.standard_normal((3, 24))
    s, rstd, y = N.rmsnorm(x, r, w, 0.1)
    assert np.allclose((y / w / s) ** -2, (s * s).mean(1, keepdims=True) + 0.1)
    dx, dw = N.rmsnorm_backward(c, s, w, rstd, r)
    h = 1e-6
    for i, j in ((0, 0), (1, 9), (2, 23)):
        d = np.zeros_like(x)
        d[i, j] = h
        num = ((c * (N.rmsnorm(x + d, r, w, 0.1)[2] - N.rmsnorm(x - d, r, w, 0.1)[2])).sum()) / (2 * h) + r[i, j]
        assert abs(num - dx[i, j]) < 1e-7
        d = np.zeros_like(w)
        d[j] = h
        assert abs((c * (N.rmsnorm(x, r, w + d, 0.1)[2] - N.rmsnorm(x, r, w - d, 0.1)[2])).sum() / (2 * h) - dw[j]) < 1e-7


# ---- workspaces -------------------------------------------------------------------------------------------------------------
def workspace_calls(L, sh, n):
    """Return codes of the entry points that take a workspace, given n bytes of it: those of the bf16 and E4M3 forms, then the FP4 ones."""
    r, lay = ctypes.byref(sh), ctypes.byref(layout())
    others = {
        "moe_route": L.moe_route(r, P, P, None, 0, P, P, P, P, n, None),
        "moe_dispatch": L.moe_dispatch(r, P, P, lay, P, P, n, None),
        "moe_expert_ffn": L.moe_expert_ffn(r, P, lay, P, P, P, P, P, P, n, None),
        "moe_expert_ffn_fp8": L.moe_expert_ffn_fp8(r, P, P, lay, P, P, P, P, P, P, P, P, P, n, None),
        "moe_combine": L.moe_combine(r, P, lay, P, P, None, P, P, n, None),
        "moe_layer": L.moe_layer(r, P, P, None, 0, P, P, P, P, None, None, None, None, P, n, None),
        "moe_layer_fp8": L.moe_layer_fp8(r, P, P, None, 0, P, P, P, P, P, P, P, None, None, None, None, P, n, None),
    }
    fp4 = {
        "moe_expert_ffn_fp4": L.moe_expert_ffn_fp4(r, P, P, lay, P, P, P, P, P, P, P, P, P, n, None),
        "moe_layer_fp4": L.moe_layer_fp4(r, P, P, None, 0, P, P, P, P, P, P, P, None, None, None, None, P, n, None),
    }
    return others, fp4


# what the bf16 and E4M3 forms use, the sum of their regions
@pytest.mark.skipif(not NO_GPU, reason="the calls are accepted, and stop where they find no device")
@pytest.mark.parametrize("dims,own", [((1, 4096, 14336, 8, 2, 2), 131072), ((4, 2048, 7168, 16, 2, 1), 238592), ((3, 4096, 4096, 8, 1, 1), 122880),
                                      ((100, 288, 160, 4, 2, 2), 268288), ((2048, 64, 96, 4, 2, 2), 2055168)], ids=str)
def test_only_the_fp4_form_asks_for_its_regions(L, dims, own):
    sh = shape(**dict(zip(("T", "d", "f", "E", "k", "G"), dims)))
    most = B.moe_workspace_bytes(sh)
    assert most > own
    others, fp4 = workspace_calls(L, sh, own)
    assert set(others.values()) == {CUDA} and set(fp4.values()) == {SMALL}, (others, fp4)
    others, _ = workspace_calls(L, sh, own - 1)
    assert set(others.values()) == {SMALL}, others
    others, fp4 = workspace_calls(L, sh, most)
    assert set(others.values()) | set(fp4.values()) == {CUDA}, (others, fp4)


@pytest.mark.parametrize("E,k,G", [(1, 1, 1), (8, 2, 2), (8, 1, 1), (16, 2, 1), (64, 6, 8), (128, 8, 8)], ids=str)
@pytest.mark.parametrize("d,f", [(64, 2048), (2048, 7168), (4096, 4096), (4096, 14336), (7168, 2048), (512, 4096)], ids=str)
def test_workspace_of_a_batch_serves_smaller_ones(L, d, f, E, k, G):
    prev = 0
    for T in [*range(0, 300), 511, 512, 1000, 2047, 2048, 4096, 16384, 65536]:
        now = B.moe_workspace_bytes(shape(T=T, d=d, f=f, E=E, k=k, G=G))
        assert now >= prev, (T, prev, now)
        prev = now


@pytest.mark.parametrize("has_lookup", [True, False])
def test_current_stream_with_and_without_the_direct_lookup(monkeypatch, has_lookup):
    """Which the calls get without a stream: the current one of the current device, also from a torch that lacks the lookup that is not public."""
    class Fake:
        cuda_stream = 4321
    monkeypatch.setattr(B, "_have_cuda", True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: Fake)
    if has_lookup:
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 1000 + device, raising=False)
    else:
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    assert B._stream(None) == (1003 if has_lookup else 4321)
    assert B._stream(Fake) == 4321


def test_lanes_of_an_epilogue_warp_of_the_fp4_products_leave_together():
    """The wait for a tile is a shuffle of the whole warp.  Were the abort word read lane by lane at the loop's head, some lanes could leave for the
    block's barrier while the others stood at the shuffle; only the wait's own result, the same in every lane, ends the loop."""
    from tests.test_boundary_cpu import enclosing_blocks, source
    for fn in ("ffn_fp4.cu", "ffn_fp4_pair.cu"):
        text = source(fn)
        waits = [m.start() for m in re.finditer(r"\bmbar_wait_warp<", text)]
        assert len(waits) == 1
        head, start, end = [b for b in enclosing_blocks(text, waits[0]) if re.search(r"\b(for|while) \(", b[0])][-1]
        assert "abort" not in head, f"{fn}: {head.strip()}"
        leaves = re.findall(r"[^;{}]*[{;]?[^;{}]*\b(?:break|return|goto)\b", text[start:end])
        assert len(leaves) == 1 and "timeout(1)" in leaves[0], leaves
        assert re.search(r"const bool go = __all_sync\(0xFFFFFFFFu, !\*abort_flag\);", text[:start])
