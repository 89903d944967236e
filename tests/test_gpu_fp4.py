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


def routed(rows_per_expert, k=1, d=128, f=128, seed=0, G=1, flags=0):
    """A batch of T tokens whose experts hold the given rows (k = 1), or T random tokens over E experts; its layout by moe_dispatch."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    if k == 1:
        E, T = len(rows_per_expert), sum(rows_per_expert)
        idx = torch.repeat_interleave(torch.arange(E, device="cuda"), torch.tensor(rows_per_expert, device="cuda")).int().view(T, 1)
        idx = idx[torch.randperm(T, generator=g, device="cuda")]
    else:
        T, E = rows_per_expert
        score = torch.rand(T, E, generator=g, device="cuda") - 0.5 * torch.arange(E, device="cuda") / E
        idx = score.topk(k, dim=1).indices.int()
        if flags & B.MOE_FLAG_SPARSE_TOPK:
            idx[torch.rand(T, k, generator=g, device="cuda") < 0.3] = -1
    shape = B.MoEShape(T, d, f, E, k, G, 0, flags)
    ws, lay = B.alloc_workspace(shape), B.alloc_layout(shape)
    x = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    xg = torch.zeros(T * min(k, G), d, device="cuda").bfloat16()
    B.moe_dispatch(shape, x, idx.contiguous(), lay, xg, ws)
    w = torch.rand(T, k, generator=g, device="cuda") + 0.1
    wt = [torch.randn(E, K, N, generator=g, device="cuda").div(K ** 0.5).bfloat16() for K, N in ((d, f), (d, f), (f, d))]
    return shape, ws, lay, x, xg, idx, w, wt


def check_ffn(shape, ws, lay, xg, w, wt, weighted=True):
    P, E = shape.T * shape.k, shape.E
    xq, sx = rows_fp4(xg)
    q = [weights_fp4(v) for v in wt]
    o = torch.full((P + 3, shape.d), 7.0, device="cuda").bfloat16()
    B.moe_expert_ffn_fp4(shape, xq, sx, lay, w if weighted else None, *[t for pair in q for t in pair], o, ws)
    assert B.moe_status(ws)[0] == 0
    off = lay.expert_offsets[: E + 1].cpu().numpy()
    n = int(off[E])
    hl = {"expert_offsets": off, "row_pair": lay.row_pair.cpu().numpy()[:n], "row_src": lay.row_src.cpu().numpy()[:n]}
    ref_w = [Q.quantize_weights(f64(v)) for v in wt]
    ref, tol = Q.expert_ffn_fp4(*Q.quantize_rows(f64(xg)), hl, w.cpu().numpy() if weighted else None, *[t for pair in ref_w for t in pair])
    got = f64(o)
    assert (np.abs(got[:n] - ref) <= tol + 2.0 ** -8 * (np.abs(ref) + tol)).all(), np.abs(got[:n] - ref).max()
    assert (got[n:] == 7.0).all()                   # rows behind the last one are left as they were
    # and not only within the allowance: nearly every row differs by the rounding of o alone
    err = np.linalg.norm(got[:n] - ref) / max(np.linalg.norm(ref), 1e-300)
    assert err <= 5e-3, err
    return o


# long walks over K with fewer tiles than SMs: their stages are shared out among the CTAs, parts of tiles are added up
@pytest.mark.parametrize("counts", [(1,), (2, 3), (0, 16, 17), (33, 1, 95), (96,), (60, 80)], ids=str)
@pytest.mark.parametrize("d,f", [(512, 4096), (4096, 512), (2080, 4640)])
def test_expert_ffn_fp4_of_shared_tiles(counts, d, f):
    shape, ws, lay, x, xg, idx, w, wt = routed(counts, d=d, f=f, seed=sum(counts) + d)
    o = check_ffn(shape, ws, lay, xg, w, wt)
    args = (shape, *rows_fp4(xg), lay, w, *quantised(wt))
    for _ in range(5):                                      # the parts are added in a fixed order, whoever is last
        again = torch.full_like(o, 7.0)
        B.moe_expert_ffn_fp4(*args, again, ws)
        assert torch.equal(again, o)


def test_expert_ffn_fp4_most_experts_and_no_token():
    shape, ws, lay, x, xg, idx, w, wt = routed((300, 1024), 4, 64, 32, 5, 8)
    check_ffn(shape, ws, lay, xg, w, wt)
    cfg = H.synth.MoEConfig("fp4-none", T=0, d=64, f=32, E=8, k=2, G=2)
    sh = B.make_shape(cfg)
    y = torch.full((1, 64), 7.0, device="cuda").bfloat16()
    wg, q = torch.zeros(64, 8, device="cuda"), quantised([v[:8].contiguous() for v in wt])
    B.moe_layer_fp4(sh, x, wg, None, *q, y, B.alloc_workspace(sh))
    assert (y == 7).all()


SMALL = [(1,), (1, 0, 3), (16, 17), (33, 1, 95, 96), (97, 192, 193), (0, 0, 5), (300,), (31, 32, 64, 65, 128, 129)]


LARGE = [(256,), (511,), (257, 300), (193, 700, 128), (1000, 0, 1, 600), (2600, 300), (385, 384, 383, 192, 320)]


@pytest.mark.parametrize("counts", LARGE, ids=str)
@pytest.mark.parametrize("d,f", [(32, 32), (256, 128), (288, 160), (512, 384), (96, 1056), (1056, 96)])
def test_expert_ffn_fp4_of_many_rows_per_expert(counts, d, f):
    shape, ws, lay, x, xg, idx, w, wt = routed(counts, d=d, f=f, seed=sum(counts) + d + f)
    check_ffn(shape, ws, lay, xg, w, wt)


@pytest.mark.parametrize("counts", SMALL, ids=str)
@pytest.mark.parametrize("d,f", [(32, 32), (256, 128), (288, 160), (512, 384), (96, 1056), (1056, 96)])
def test_expert_ffn_fp4_by_rows_per_expert(counts, d, f):
    shape, ws, lay, x, xg, idx, w, wt = routed(counts, d=d, f=f, seed=sum(counts) + d + f)
    check_ffn(shape, ws, lay, xg, w, wt)


@pytest.mark.parametrize("T,E,k,G,d,f", [(5, 4, 2, 2, 64, 96), (200, 16, 4, 4, 320, 416), (700, 8, 3, 8, 512, 256), (64, 128, 8, 8, 128, 64),
                                         (1500, 6, 2, 3, 288, 544)])
@pytest.mark.parametrize("flags", [0, B.MOE_FLAG_WEIGHT_IN_COMBINE, B.MOE_FLAG_SPARSE_TOPK], ids=["plain", "weight-in-combine", "sparse"])
def test_expert_ffn_fp4_routed(T, E, k, G, d, f, flags):
    shape, ws, lay, x, xg, idx, w, wt = routed((T, E), k, d, f, T, G, flags)
    check_ffn(shape, ws, lay, xg, w, wt, weighted=not flags & B.MOE_FLAG_WEIGHT_IN_COMBINE)


def quantised(wt):
    return [t for v in wt for t in weights_fp4(v)]


@pytest.mark.parametrize("T,E,k,G,d,f,score", [(1, 4, 2, 2, 64, 32, 0), (50, 16, 4, 4, 320, 416, 1), (900, 8, 2, 8, 512, 256, 0), (333, 128, 8, 8, 96, 160, 1)])
@pytest.mark.parametrize("flags", [0, B.MOE_FLAG_WEIGHT_IN_COMBINE], ids=["plain", "weight-in-combine"])
def test_layer_fp4_matches_its_oracle(T, E, k, G, d, f, score, flags):
    cfg = H.synth.MoEConfig("fp4", T=T, d=d, f=f, E=E, k=k, G=G, score_fn=score, seed=T + E)
    run = H.Run(cfg, flags)
    t = run.t
    wt = [t["w1"], t["w3"], t["w2"]]
    lay_dev = B.alloc_layout(run.shape)
    for _ in range(2):
        run.y.fill_(3.0)
        B.moe_layer_fp4(run.shape, t["x"], t["w_gate"], t["bias"], *quantised(wt), run.y, run.ws, logits=run.logits, topk_idx=run.idx,
                        topk_w=run.w, layout=lay_dev)
    assert run.status()[0] == 0
    run.lay = lay_dev
    idx_ref, _ = H.check_route(run)          # routing runs on the bf16 activations, as in moe_layer
    lay = H.check_layout(run, idx_ref)
    # quantising commutes with the dispatch copy: quantise x, then take the dispatched rows
    xq, sx = Q.quantize_rows(f64(t["x"]))
    dt = lay["disp_token"].astype(np.int64)
    ref_w = [v for w in wt for v in Q.quantize_weights(f64(w))]
    in_combine = bool(flags & B.MOE_FLAG_WEIGHT_IN_COMBINE)
    o_ref, _ = Q.expert_ffn_fp4(xq[dt], sx[dt], lay, None if in_combine else run.host_w(), *ref_w)
    _, _, y_ref = O.combine(o_ref, lay, idx_ref, run.host_w() if in_combine else None, E, G)
    H.assert_close_out(f64(run.y)[:T], y_ref, "fp4 layer y")


def test_layer_fp4_is_its_stages():
    """moe_layer_fp4 against moe_route, moe_dispatch, moe_quantize_rows_fp4, moe_expert_ffn_fp4 and moe_combine: the same bits."""
    cfg = H.synth.MoEConfig("fp4-stages", T=257, d=288, f=352, E=12, k=3, G=4, seed=8)
    run = H.Run(cfg)
    t, q = run.t, quantised([run.t["w1"], run.t["w3"], run.t["w2"]])
    y = torch.zeros_like(run.y)
    B.moe_layer_fp4(run.shape, t["x"], t["w_gate"], t["bias"], *q, y, run.ws)
    run.route()
    run.dispatch()
    B.moe_expert_ffn_fp4(run.shape, *rows_fp4(run.xg), run.lay, run.w, *q, run.o, run.ws)
    run.combine()
    assert torch.equal(run.y, y)


def test_norm_then_fp4_layer_then_norm():
    """A transformer block's MoE half, as it is used: norm with the residual, the layer on its output, the next block's norm."""
    cfg = H.synth.MoEConfig("fp4-block", T=130, d=256, f=288, E=8, k=2, G=2, seed=5)
    run = H.Run(cfg)
    t, q = run.t, quantised([run.t["w1"], run.t["w3"], run.t["w2"]])
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
    stream, attn = rnd(130, 256).bfloat16(), rnd(130, 256).bfloat16()
    w = 1 + 0.1 * rnd(256)
    y, out = torch.zeros_like(attn), torch.zeros_like(attn)
    s0, a0 = f64(stream), f64(attn)
    B.moe_rmsnorm(attn, w, 1e-6, y=y, residual=stream, res_out=stream)
    B.moe_layer_fp4(run.shape, y, t["w_gate"], t["bias"], *q, run.y, run.ws, logits=run.logits, topk_idx=run.idx, topk_w=run.w)
    final = torch.zeros_like(y)
    B.moe_rmsnorm(run.y, w, 1e-6, y=final, residual=stream, res_out=out)
    from oracle import norm_oracle as N
    s, _, y_ref = N.rmsnorm(s0, a0, f64w := w.double().cpu().numpy(), 1e-6)
    assert np.abs(f64(y) - y_ref).max() <= 2.0 ** -8 * np.abs(y_ref).max() + 1e-5
    idx = run.host_idx()
    lay = O.layout(idx, 8, 2)
    xq, sx = Q.quantize_rows(f64(y))
    dt = lay["disp_token"].astype(np.int64)
    o_ref, _ = Q.expert_ffn_fp4(xq[dt], sx[dt], lay, run.host_w(), *[v for n in ("w1", "w3", "w2") for v in Q.quantize_weights(f64(t[n]))])
    _, _, m_ref = O.combine(o_ref, lay, idx, None, 8, 2)
    H.assert_close_out(f64(run.y)[:130], m_ref, "layer")
    s2, _, f_ref = N.rmsnorm(m_ref, f64(stream), f64w, 1e-6)
    H.assert_close_out(f64(out), s2, "stream")
    H.assert_close_out(f64(final), f_ref, "next norm")


def test_norm_feeds_fp8_experts():
    """yq / scale of the norm are the operand of moe_expert_ffn_fp8 (one group: dispatched row = token)."""
    from oracle import fp8_oracle as F
    cfg = H.synth.MoEConfig("fp8-norm", T=200, d=256, f=384, E=8, k=2, G=1, seed=6)
    run = H.Run(cfg)
    t = run.t
    w = (1 + 0.1 * torch.randn(256, device="cuda")).bfloat16()
    y, yq, sc = torch.zeros_like(t["x"]), torch.zeros(200, 256, dtype=torch.uint8, device="cuda"), torch.zeros(200, device="cuda")
    B.moe_rmsnorm(t["x"], w, 1e-6, y=y, yq=yq, scale=sc)
    B.moe_route(run.shape, y, t["w_gate"], t["bias"], run.logits, run.idx, run.w, run.ws)
    B.moe_dispatch(run.shape, None, run.idx, run.lay, None, run.ws)
    wq = []
    for name in ("w1", "w3", "w2"):
        E, K, N = t[name].shape
        wq += [torch.zeros(E, N, K, dtype=torch.uint8, device="cuda"), torch.zeros(E, N, device="cuda")]
        B.moe_quantize_weights(t[name], *wq[-2:])
    B.moe_expert_ffn_fp8(run.shape, yq, sc, run.lay, run.w, *wq, run.o, run.ws)
    assert run.status()[0] == 0
    lay = O.layout(run.host_idx(), 8, 1)
    ref = F.expert_ffn_fp8(yq.cpu().numpy(), sc.cpu().numpy(), lay, run.host_w(), *[v.cpu().numpy() for v in wq])
    H.assert_close_out(f64(run.o)[: cfg.P], ref, "fp8 experts on the norm's codes")


def test_expert_ffn_fp4_captured_on_two_streams_and_with_an_empty_batch():
    shape, ws, lay, x, xg, idx, w, wt = routed((150, 8), 2, 256, 288, 3)
    q, (xq, sx) = quantised(wt), rows_fp4(xg)
    want = torch.zeros(300, 256, device="cuda").bfloat16()
    B.moe_expert_ffn_fp4(shape, xq, sx, lay, w, *q, want, ws)
    side = [torch.cuda.Stream() for _ in range(2)]
    outs, graphs = [torch.zeros_like(want) for _ in side], []
    wss = [ws, B.alloc_workspace(shape)]                     # calls that may overlap have a workspace each
    for s, o, v in zip(side, outs, wss):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            B.moe_expert_ffn_fp4(shape, xq, sx, lay, w, *q, o, v)
        graphs.append(graph)
    torch.cuda.synchronize()
    for _ in range(3):
        for s, graph in zip(side, graphs):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    empty = B.MoEShape(0, 256, 288, 8, 2, 1, 0, 0)
    B.moe_expert_ffn_fp4(empty, xq, sx, lay, w, *q, want, ws)
    assert torch.equal(outs[0], want)


def test_fp4_a_nan_block_reaches_its_own_rows_and_columns_only():
    shape, ws, lay, x, xg, idx, w, wt = routed((40, 30), d=128, f=96, seed=2)
    xg[int(lay.row_src[3]), 5] = float("inf")               # a row of the first expert
    wt[2][1, 7, 11] = float("nan")                            # column 11 of the second expert's W2
    q, (xq, sx) = quantised(wt), rows_fp4(xg)
    o = torch.zeros(70, 128, device="cuda").bfloat16()
    B.moe_expert_ffn_fp4(shape, xq, sx, lay, w, *q, o, ws)
    bad = torch.isnan(o)
    want = torch.zeros_like(bad)
    want[3] = True
    want[40:, 11] = True
    assert torch.equal(bad, want)


def test_expert_ffn_fp4_reports_a_source_row_out_of_range():
    shape, ws, lay, x, xg, idx, w, wt = routed((10, 20), d=64, f=64, seed=1)
    lay.row_src[4] = 30
    o = torch.zeros(30, 64, device="cuda").bfloat16()
    B.moe_expert_ffn_fp4(shape, *rows_fp4(xg), lay, w, *quantised(wt), o, ws)
    st = B.moe_status(ws)
    assert st[0] == B.MOE_DEV_INDEX_OUT_OF_RANGE and st[2] == 30 and st[3] == 4


class Fenced:
    """Buffers of exactly the size that the interface asks for, in the middle of bytes that nothing may touch."""

    def __init__(self):
        self.all = []

    def __call__(self, nbytes, dtype=torch.uint8, shape=None, fill=0):
        pad = 1 << 16
        raw = torch.full((nbytes + 2 * pad,), 0xC5, dtype=torch.uint8, device="cuda")
        assert raw.data_ptr() % 128 == 0
        raw[pad:pad + nbytes] = fill
        self.all.append((raw, pad, nbytes))
        t = raw[pad:pad + nbytes].view(dtype)
        return t if shape is None else t.view(shape)

    def check(self):
        torch.cuda.synchronize()
        for raw, pad, n in self.all:
            assert (raw[:pad] == 0xC5).all() and (raw[pad + n:] == 0xC5).all()


@pytest.mark.parametrize("T,E,k,d,f,zipf", [(1, 8, 2, 2048, 4096, 0), (3, 64, 8, 96, 64, 0), (97, 4, 1, 288, 544, 0), (129, 1, 1, 32, 32, 0), (700, 4, 2, 288, 160, 1),
                                            (2000, 16, 1, 64, 96, 1), (640, 128, 5, 32, 32, 1), (1537, 3, 3, 96, 1056, 0), (500, 2, 1, 160, 288, 0)])
def test_fp4_stays_inside_its_buffers(T, E, k, d, f, zipf):
    g = torch.Generator(device="cuda").manual_seed(T)
    idx = (torch.rand(T, E, generator=g, device="cuda") - zipf * torch.arange(E, device="cuda") / E).topk(k, dim=1).indices.int().contiguous()
    shape, buf = B.MoEShape(T, d, f, E, k, 1, 0, 0), Fenced()
    lay, ws = B.alloc_layout(shape), buf(B.moe_workspace_bytes(shape))
    x = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    B.moe_dispatch(shape, None, idx, lay, None, ws)
    w = torch.rand(T, k, generator=g, device="cuda") + 0.1
    q, refs = [], []
    for K, N in ((d, f), (d, f), (f, d)):
        v = torch.randn(E, K, N, generator=g, device="cuda").div(K ** 0.5).bfloat16()
        q += [buf(E * N * K // 2, shape=(E, N, K // 2)), buf(B.moe_fp4_scale_bytes(E, K, N))]
        B.moe_quantize_weights_fp4(v, *q[-2:])
        back = buf(E * K * N * 2, torch.bfloat16, (E, K, N))
        B.moe_dequantize_weights_fp4(*q[-2:], back)
        refs += Q.quantize_weights(f64(v))
    xq, sx = buf(T * d // 2, shape=(T, d // 2)), buf(T * d // 32, shape=(T, d // 32))
    B.moe_quantize_rows_fp4(x, xq, sx)
    B.moe_dequantize_rows_fp4(xq, sx, buf(T * d * 2, torch.bfloat16, (T, d)))
    o = buf(T * k * d * 2, torch.bfloat16, (T * k, d))
    ws[64:] = 0xEE                                           # nothing in the workspace but the status block has to start at zero
    B.moe_expert_ffn_fp4(shape, xq, sx, lay, w, *q, o, ws)
    assert B.moe_status(ws)[0] == 0
    buf.check()
    n = T * k
    hl = {"expert_offsets": lay.expert_offsets[: E + 1].cpu().numpy(), "row_pair": lay.row_pair.cpu().numpy()[:n], "row_src": lay.row_src.cpu().numpy()[:n]}
    ref, tol = Q.expert_ffn_fp4(*Q.quantize_rows(f64(x)), hl, w.cpu().numpy(), *refs)
    got = f64(o)
    assert (np.abs(got - ref) <= tol + 2.0 ** -8 * (np.abs(ref) + tol)).all()
    # the same through the layer, with its own routing
    wg, y = torch.randn(d, E, generator=g, device="cuda") * 0.1, buf(T * d * 2, torch.bfloat16, (T, d), fill=0xFF)
    B.moe_layer_fp4(shape, x, wg, None, *q, y, ws)
    assert B.moe_status(ws)[0] == 0 and torch.isfinite(y.float()).all()
    buf.check()


@pytest.mark.parametrize("rows,cols", [(1, 8), (3, 520), (700, 1024), (61, 2056), (9, 16384), (2500, 4096)])
def test_norm_stays_inside_its_buffers(rows, cols):
    buf = Fenced()
    bf = lambda: buf(rows * cols * 2, torch.bfloat16, (rows, cols))   # noqa: E731
    x, r, dy = (torch.randn(rows, cols, device="cuda").bfloat16() for _ in range(3))
    w = torch.ones(cols, device="cuda")
    y, s, q = bf(), bf(), buf(rows * cols, shape=(rows, cols))
    sc, rs = buf(rows * 4, torch.float32), buf(rows * 4, torch.float32)
    B.moe_rmsnorm(x, w, 1e-6, y=y, residual=r, res_out=s, yq=q, scale=sc, rstd=rs)
    dx, dw = bf(), buf(cols * 4, torch.float32)
    B.moe_rmsnorm_backward(dy, s, w, rs, dx, dw, buf(B.moe_rmsnorm_backward_workspace_bytes(rows, cols), fill=0xEE), dres=r)
    buf.check()
    assert torch.isfinite(dx.float()).all() and torch.isfinite(dw).all()


@pytest.mark.parametrize("row,pair", [(4, 1 << 30), (4, 30), (7, -1), (29, -(1 << 31))])
def test_expert_ffn_fp4_reports_a_pair_out_of_range(row, pair):
    """The gate weight is not read with a pair that is not in the batch; the other rows are those of a sound layout."""
    shape, ws, lay, x, xg, idx, w, wt = routed((10, 20), d=64, f=64, seed=1)
    q, rows = quantised(wt), rows_fp4(xg)
    want, o = (torch.zeros(30, 64, device="cuda").bfloat16() for _ in range(2))
    B.moe_expert_ffn_fp4(shape, *rows, lay, w, *q, want, ws)
    lay.row_pair[row] = pair
    B.moe_expert_ffn_fp4(shape, *rows, lay, w, *q, o, ws)
    st = B.moe_status(ws)
    assert st[0] == B.MOE_DEV_INDEX_OUT_OF_RANGE and st[2] == pair and st[3] == row
    keep = torch.arange(30, device="cuda") != row
    assert torch.equal(o[keep], want[keep])


# ---- sizes at which the kernels' loops come round again --------------------------------------------------------------------------
def test_rows_fp4_beyond_one_pass_of_the_grid():
    """The grid takes 16 blocks per SM x 8192 values at once (19.4 M on 148 SMs): 2.1 times as many, against calls of 1000 rows, which one pass takes."""
    cols = 2880
    rows = int(2.1 * 16 * torch.cuda.get_device_properties(0).multi_processor_count * 8192) // cols + 1
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(rows, cols, generator=g, device="cuda").mul_(torch.exp2(8 * torch.rand(rows, 1, generator=g, device="cuda"))).bfloat16()
    q, s = rows_fp4(x)
    back = torch.full_like(x, 7.0)
    B.moe_dequantize_rows_fp4(q, s, back)
    for i in range(0, rows, 1000):
        qi, si = rows_fp4(x[i:i + 1000])
        bi = torch.full_like(x[i:i + 1000], 7.0)
        B.moe_dequantize_rows_fp4(qi, si, bi)
        assert torch.equal(q[i:i + 1000], qi) and torch.equal(s[i:i + 1000], si) and torch.equal(back[i:i + 1000], bi), i
    q_ref, s_ref = Q.quantize_rows(f64(x[-300:]))
    assert np.array_equal(q[-300:].cpu().numpy(), q_ref) and np.array_equal(s[-300:].cpu().numpy(), s_ref)


def with_empty_experts(T, E, k, d, f, flags=0, seed=0):
    """T tokens over E experts, of which every fifth and the first and last two get none; the others' rows fall off from expert to expert."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    score = torch.rand(T, E, generator=g, device="cuda") - 0.6 * torch.arange(E, device="cuda") / E
    score[:, ::5] = score[:, :2] = score[:, -2:] = -9
    idx = score.topk(k, dim=1).indices.int()
    if flags & B.MOE_FLAG_SPARSE_TOPK:
        idx[torch.rand(T, k, generator=g, device="cuda") < 0.03] = -1
    shape = B.MoEShape(T, d, f, E, k, 1, 0, flags)
    ws, lay = B.alloc_workspace(shape), B.alloc_layout(shape)
    x = torch.randn(T, d, generator=g, device="cuda").mul_(torch.exp2(4 * torch.rand(T, 1, generator=g, device="cuda"))).bfloat16()
    B.moe_dispatch(shape, None, idx.contiguous(), lay, None, ws)
    w = torch.rand(T, k, generator=g, device="cuda") + 0.1
    wt = [torch.randn(E, K, N, generator=g, device="cuda").div(K ** 0.5).bfloat16() for K, N in ((d, f), (d, f), (f, d))]
    return shape, ws, lay, x, w, wt


# from 512 rows per SM on (75776 on 148 SMs) a warp of the sorting kernel takes four rows: experts begin and end inside them, tiles do, and the last warp has
# fewer.  64 experts: CTA pairs, tiles of 256 and 208 rows; 1024 experts: single CTAs, tiles of 96.
@pytest.mark.parametrize("T,E,k,d,f", [(20011, 64, 4, 64, 96), (20011, 1024, 4, 64, 32), (40003, 96, 2, 288, 64)])
@pytest.mark.parametrize("flags", [0, B.MOE_FLAG_SPARSE_TOPK], ids=["plain", "sparse"])
def test_expert_ffn_fp4_of_more_pairs_than_warps(T, E, k, d, f, flags):
    assert T * k * 0.95 >= 512 * torch.cuda.get_device_properties(0).multi_processor_count
    shape, ws, lay, x, w, wt = with_empty_experts(T, E, k, d, f, flags, T + E)
    off = lay.expert_offsets[: E + 1].cpu().numpy()
    assert (np.diff(off) == 0).sum() >= E // 5 and (off[1:] % 4 != 0).any() and (off[-1] < T * k) == (flags != 0)
    check_ffn(shape, ws, lay, x, w, wt)


# Every cluster (CTA) walks its pipeline round several times (six stages; single CTAs four) and comes to its accumulators a third time.  Pairs: GEMM-1 has 15 x 25
# tiles of 9 stages, GEMM-2 19 x 9 of 13, for at most 74 clusters.  Single CTAs: 704 tiles of 6 stages, 384 of 6, for 148.
@pytest.mark.parametrize("counts,d,f", [((1500, 700, 1300), 2080, 3104), ((0, 1029, 2100, 1), 3104, 1312), ((20, 19, 21, 23) * 16, 1312, 1312),
                                        ((70, 0, 97, 33) * 16, 1056, 1312)], ids=["pairs", "pairs-2", "single", "single-2"])
def test_expert_ffn_fp4_when_the_pipeline_comes_round(counts, d, f):
    shape, ws, lay, x, xg, idx, w, wt = routed(counts, d=d, f=f, seed=len(counts) + d)
    o = check_ffn(shape, ws, lay, xg, w, wt)
    again = torch.full_like(o, 7.0)
    B.moe_expert_ffn_fp4(shape, *rows_fp4(xg), lay, w, *quantised(wt), again, ws)
    assert torch.equal(again, o)


@pytest.mark.parametrize("T,E,k,G,d,f,score", [(3001, 16, 4, 4, 1056, 1312, 0), (1500, 64, 6, 8, 1312, 1056, 1), (9, 8, 2, 2, 4096, 2080, 0)])
def test_layer_fp4_is_its_stages_at_size(T, E, k, G, d, f, score):
    """The layer against its stages, bit for bit, eagerly and replayed from a graph with other tokens."""
    cfg = H.synth.MoEConfig("fp4-size", T=T, d=d, f=f, E=E, k=k, G=G, score_fn=score, seed=T)
    run = H.Run(cfg)
    t, q = run.t, quantised([run.t["w1"], run.t["w3"], run.t["w2"]])
    y = torch.zeros_like(run.y)

    def stages():
        run.route()
        run.dispatch()
        B.moe_expert_ffn_fp4(run.shape, *rows_fp4(run.xg), run.lay, run.w, *q, run.o, run.ws)
        run.combine()
        return run.y.clone()

    want = stages()
    B.moe_layer_fp4(run.shape, t["x"], t["w_gate"], t["bias"], *q, y, run.ws)
    assert torch.equal(want, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.moe_layer_fp4(run.shape, t["x"], t["w_gate"], t["bias"], *q, y, run.ws)
    t["x"].copy_(torch.randn(T, d, generator=torch.Generator(device="cuda").manual_seed(9), device="cuda"))
    for _ in range(3):
        y.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert run.status()[0] == 0 and torch.equal(stages(), y)


@pytest.mark.parametrize("d,f,E,k", [(512, 4096, 8, 2), (4096, 2048, 4, 1), (2048, 1024, 16, 2)])
def test_fp4_workspace_of_a_batch_serves_smaller_ones(d, f, E, k):
    """One workspace, allocated for the largest batch, for every smaller one, with the bits that a workspace of its own gives."""
    g = torch.Generator(device="cuda").manual_seed(d)
    wt = [torch.randn(E, K, N, generator=g, device="cuda").div(K ** 0.5).bfloat16() for K, N in ((d, f), (d, f), (f, d))]
    q, wg = quantised(wt), torch.randn(d, E, generator=g, device="cuda") * 0.1
    ws = B.alloc_workspace(B.MoEShape(600, d, f, E, k, 1, 0, 0))
    ws[64:] = 0xEE
    for T in (600, 97, 16, 3, 2, 1, 40, 600):
        x = torch.randn(T, d, generator=g, device="cuda").bfloat16()
        shape = B.MoEShape(T, d, f, E, k, 1, 0, 0)
        y, want = torch.zeros_like(x), torch.zeros_like(x)
        B.moe_layer_fp4(shape, x, wg, None, *q, y, ws)
        B.moe_layer_fp4(shape, x, wg, None, *q, want, B.alloc_workspace(shape))
        assert B.moe_status(ws)[0] == 0 and torch.equal(y, want), T


@pytest.mark.parametrize("counts,d,f", [((3, 0, 20), 512, 4096), ((70, 33, 97), 288, 352), ((700, 300, 90), 288, 352)], ids=["shared", "single", "pairs"])
def test_expert_ffn_fp4_on_an_aborted_workspace_ends(counts, d, f):
    """The abort word of a wait that gave up makes the products skip their work; once it is reset the call gives the same bits as before."""
    shape, ws, lay, x, xg, idx, w, wt = routed(counts, d=d, f=f, seed=d)
    want = check_ffn(shape, ws, lay, xg, w, wt)
    args = (shape, *rows_fp4(xg), lay, w, *quantised(wt))
    o = torch.full_like(want, 7.0)
    B.moe_selftest_wait_timeout(ws, 300_000)
    B.moe_expert_ffn_fp4(*args, o, ws)
    st = B.moe_status(ws)
    assert st[0] == B.MOE_DEV_TIMEOUT and st[1] == 9 and st[4] == 1, st
    assert (o == 7).all()
    B.moe_status_reset(ws)
    B.moe_expert_ffn_fp4(*args, o, ws)
    assert B.moe_status(ws)[0] == 0 and torch.equal(o, want)


# ---- offsets that pass 32 bits: the last part of a large call against a small call on that part alone --------------------------------
def test_norm_and_rows_fp4_past_32_bits():
    rows, cols, tail = (1 << 20) + 4099, 4096, 5000              # 4.3e9 elements
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w, y, rstd = torch.ones(cols, device="cuda"), torch.empty_like(x), torch.empty(rows, device="cuda")
    B.moe_rmsnorm(x, w, 1e-6, y=y, rstd=rstd)
    y2, rstd2 = torch.empty_like(x[-tail:]), torch.empty(tail, device="cuda")
    B.moe_rmsnorm(x[-tail:], w, 1e-6, y=y2, rstd=rstd2)
    assert torch.equal(y[-tail:], y2) and torch.equal(rstd[-tail:], rstd2)
    dy = y                                                        # dx over dy
    dx2, dw, ws = torch.empty_like(y2), torch.empty(cols, device="cuda"), torch.empty(B.moe_rmsnorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.moe_rmsnorm_backward(y2, x[-tail:], w, rstd2, dx2, dw, ws)
    B.moe_rmsnorm_backward(dy, x, w, rstd, dy, dw, ws)
    assert torch.equal(dy[-tail:], dx2)
    q, s = rows_fp4(x)
    q2, s2 = rows_fp4(x[-tail:])
    assert torch.equal(q[-tail:], q2) and torch.equal(s[-tail:], s2)
    back, back2 = y, torch.empty_like(y2)
    B.moe_dequantize_rows_fp4(q, s, back)
    B.moe_dequantize_rows_fp4(q2, s2, back2)
    assert torch.equal(back[-tail:], back2)
    del x, y, dy, back, q
    torch.cuda.empty_cache()


def test_weights_fp4_past_32_bits():
    E, K, N = 300, 7168, 2048                                     # 4.4e9 elements
    w = torch.empty(E, K, N, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(2))
    q, s = weights_fp4(w)
    q2, s2 = weights_fp4(w[-2:])
    assert torch.equal(q[-2:], q2) and torch.equal(s.view(E, -1)[-2:], s2.view(2, -1))
    back2 = torch.empty_like(w[-2:])
    B.moe_dequantize_weights_fp4(q2, s2, back2)
    B.moe_dequantize_weights_fp4(q, s, w)
    assert torch.equal(w[-2:], back2)
    del w, q
    torch.cuda.empty_cache()


def test_expert_ffn_fp4_past_32_bits():
    """1.1 M pairs of 4096 columns (o has 4.5e9 elements); the last tokens alone give the same rows."""
    T, E, k, d, f, tail = 138000, 8, 8, 4096, 64, 3001
    g = torch.Generator(device="cuda").manual_seed(3)
    wt = [torch.randn(E, K, N, generator=g, device="cuda").div(K ** 0.5).bfloat16() for K, N in ((d, f), (d, f), (f, d))]
    q = quantised(wt)
    x = torch.empty(T, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    idx = torch.rand(T, E, generator=g, device="cuda").topk(k, dim=1).indices.int().contiguous()
    w = torch.rand(T, k, generator=g, device="cuda") + 0.1
    out = []
    for n in (slice(0, T), slice(T - tail, T)):
        xs, ids, ws_ = x[n].contiguous(), idx[n].contiguous(), w[n].contiguous()
        shape = B.MoEShape(xs.shape[0], d, f, E, k, 1, 0, 0)
        lay, ws = B.alloc_layout(shape), B.alloc_workspace(shape)
        B.moe_dispatch(shape, None, ids, lay, None, ws)
        o = torch.full((xs.shape[0] * k, d), 7.0, dtype=torch.bfloat16, device="cuda")
        B.moe_expert_ffn_fp4(shape, *rows_fp4(xs), lay, ws_, *q, o, ws)
        assert B.moe_status(ws)[0] == 0
        out.append(o[lay.pair_row.view(-1, k)[-tail:].long().flatten()])
        del o, ws
    assert torch.equal(*out)
    torch.cuda.empty_cache()
