"""The norm of the residual stream and its gradients against float64, through the C ABI."""
import numpy as np
import pytest
import torch

from oracle import norm_oracle as N
from paper_2605_05607_b200 import binding as B

pytestmark = pytest.mark.gpu

U32, U16 = 2.0 ** -24, 2.0 ** -8      # half a step of fp32 and of bf16, relative
EPS = 1e-6
# fp32 roundings on the longest way to a row's sum: 64 terms per thread, 5 + 16 partial sums, and one each for s, its square, the mean, eps
# and the root (which halves what comes before it)
CHAIN = 64 + 21 + 5


def f64(t):
    return t.double().cpu().numpy()


def make(rows, cols, seed, res=True, w32=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
    x = rnd(rows, cols).bfloat16()
    r = (rnd(rows, cols) * 3).bfloat16() if res else None
    w = 1 + 0.3 * rnd(cols)
    return x, r, (w if w32 else w.bfloat16())


def e4m3(codes):
    return f64(codes.view(torch.float8_e4m3fn).float())


def check_forward(x, r, w, out, eps=EPS):
    s, rstd, y = N.rmsnorm(f64(x), None if r is None else f64(r), f64(w), eps)
    assert (np.abs(f64(out["rstd"]) - rstd) <= CHAIN * U32 * rstd).all()
    y_err = (CHAIN + 4) * U32 * np.abs(y)
    if "res" in out:
        assert (np.abs(f64(out["res"]) - s) <= (U16 + U32) * np.abs(s)).all()
    if "y" in out:
        assert (np.abs(f64(out["y"]) - y) <= U16 * np.abs(y) + (1 + U16) * y_err).all()
    if "q" in out:
        top = np.abs(y).max(axis=1)
        sc = f64(out["scale"])
        ref = np.where(top == 0, 1.0, top / 448)
        assert (np.abs(sc - ref) <= (CHAIN + 6) * U32 * ref).all()
        # half a step of E4M3: 2^-4 of a normal value, 2^-10 of the scale below 2^-6
        got = e4m3(out["q"]) * sc[:, None]
        assert (np.abs(got - y) <= (2.0 ** -4 + 2.0 ** -18) * np.abs(y) + 2.0 ** -10 * sc[:, None]).all()


def forward(x, r, w, y=True, q=True, eps=EPS, keep=True):
    rows, cols = x.shape
    out = {"rstd": torch.full((rows,), 7.0, device="cuda")}
    if y:
        out["y"] = torch.full_like(x, 7.0)
    if q:
        out["q"] = torch.full((rows, cols), 9, dtype=torch.uint8, device="cuda")
        out["scale"] = torch.full((rows,), 7.0, device="cuda")
    if r is not None and keep:
        out["res"] = torch.full_like(x, 7.0)
    B.moe_rmsnorm(x, w, eps, y=out.get("y"), residual=r, res_out=out.get("res"), yq=out.get("q"), scale=out.get("scale"),
                  rstd=out["rstd"])
    return out


COLS = [8, 16, 248, 256, 264, 512, 520, 1024, 1032, 2048, 2056, 2880, 4096, 4104, 7168, 8192, 8200, 16384]


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("rows", [1, 7, 300])
def test_norm_matches_float64(rows, cols):
    for i, (res, y, q, w32) in enumerate([(True, True, True, False), (False, True, False, True), (True, False, True, True),
                                          (False, False, True, False), (True, True, False, False), (False, True, True, True)]):
        x, r, w = make(rows, cols, 100 * rows + cols + i, res, w32)
        check_forward(x, r, w, forward(x, r, w, y, q))


def test_norm_of_many_rows():
    """More rows than blocks, so that each takes several."""
    for cols in (64, 640, 1536, 4096):
        x, r, w = make(9001, cols, cols)
        check_forward(x, r, w, forward(x, r, w))


def test_norm_in_place_and_without_the_optional_outputs():
    x, r, w = make(50, 2880, 3)
    want = forward(x, r, w)
    stream, y = r.clone(), x.clone()
    B.moe_rmsnorm(y, w, EPS, y=y, residual=stream, res_out=stream)          # y over x, the stream over itself
    assert torch.equal(y, want["y"]) and torch.equal(stream, want["res"])
    stream, y = x.clone(), r.clone()
    B.moe_rmsnorm(stream, w, EPS, y=y, residual=y, res_out=stream)          # y over the residual, the sum over x
    assert torch.equal(y, want["y"]) and torch.equal(stream, want["res"])
    out = forward(x, r, w, keep=False)
    assert torch.equal(out["y"], want["y"]) and torch.equal(out["q"], want["q"])


def test_norm_rows_of_extreme_values():
    cols = 512
    x = torch.zeros(8, cols, device="cuda").bfloat16()
    w = torch.ones(cols, device="cuda")
    x[1] = 1e-20                       # vanishes against eps
    x[2, 5] = 1e18                     # one huge value: everything else underflows
    x[3] = 2.0 ** -133                 # the least subnormal
    x[4, 0], x[5, 0], x[6, 0] = float("nan"), float("inf"), -float("inf")
    x[7] = 3.0
    out = forward(x, None, w)
    keep = [0, 1, 2, 3, 7]
    check_forward(x[keep], None, w, {n: t[keep] for n, t in out.items()})
    assert (e4m3(out["q"])[0] == 0).all() and out["scale"][0].item() == 1.0
    for row in (4, 5, 6):
        assert torch.isnan(out["y"][row]).any() and torch.isnan(out["scale"][row])
        assert np.isnan(e4m3(out["q"])[row]).all()
    assert torch.isnan(out["y"][4]).all()
    zero = forward(x[:1], None, w, eps=0.0)   # 0 / 0
    assert torch.isnan(zero["y"]).all()
    # values so small that the scale itself vanishes: codes of zero, not of infinity
    tiny = forward(x[7:8], None, torch.full((cols,), 2.0 ** -148, device="cuda"))
    assert tiny["scale"].item() == 1.0 and (e4m3(tiny["q"]) == 0).all()


def test_norm_of_no_rows_and_untouched_neighbours():
    w = torch.ones(256, device="cuda")
    pad = torch.full((3, 256), 5.0, device="cuda").bfloat16()
    B.moe_rmsnorm(pad[:0], w, EPS, y=pad[:0])
    x, r, _ = make(5, 256, 1)
    y, sc, rs = torch.full((7, 256), 5.0, device="cuda").bfloat16(), torch.full((7,), 5.0, device="cuda"), torch.full((7,), 5.0, device="cuda")
    q = torch.full((7, 256), 5, dtype=torch.uint8, device="cuda")
    B.moe_rmsnorm(x, w, EPS, y=y[1:6], residual=r, yq=q[1:6], scale=sc[1:6], rstd=rs[1:6])
    torch.cuda.synchronize()
    assert (pad == 5).all()
    for t in (y, q, sc, rs):
        assert (t[0] == 5).all() and (t[6] == 5).all() and not (t[1:6] == 5).all()


def check_backward(dy, s, w, rstd, skip, dx, dw):
    rows, cols = dy.shape
    a, sv, wv, rv = f64(dy), f64(s), f64(w), f64(rstd)
    k = None if skip is None else f64(skip)
    dx_ref, dw_ref = N.rmsnorm_backward(a, sv, wv, rv, k)
    xhat, g = sv * rv[:, None], a * wv
    # every term of dx passes a handful of roundings, those of the mean up to CHAIN
    mag = rv[:, None] * (6 * np.abs(g) + np.abs(xhat) * (CHAIN + 6) * np.abs(g * xhat).mean(axis=1, keepdims=True))
    err = U32 * (mag + np.abs(dx_ref) + (0 if k is None else np.abs(k)))
    assert (np.abs(f64(dx) - dx_ref) <= U16 * np.abs(dx_ref) + (1 + U16) * err).all()
    # dw: additions in a row inside a block, then over a warp's share of the blocks, then over eight warps
    depth = -(-rows // 592) + 592 // 8 + 8 + 4
    assert (np.abs(f64(dw) - dw_ref) <= depth * U32 * np.abs(a * xhat).sum(axis=0) + 1e-300).all()


def backward(dy, s, w, rstd, skip=None):
    rows, cols = dy.shape
    dx, dw = torch.full_like(dy, 7.0), torch.full((cols,), 7.0, device="cuda")
    ws = torch.full((B.moe_rmsnorm_backward_workspace_bytes(rows, cols),), 255, dtype=torch.uint8, device="cuda")
    B.moe_rmsnorm_backward(dy, s, w, rstd, dx, dw, ws, dres=skip)
    return dx, dw


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("rows", [1, 5, 700])
def test_norm_backward_matches_float64(rows, cols):
    for skip, w32 in ((True, False), (False, True)):
        x, r, w = make(rows, cols, rows + cols, True, w32)
        out = forward(x, r, w, q=False)
        g = torch.Generator(device="cuda").manual_seed(rows)
        dy = torch.randn(rows, cols, generator=g, device="cuda").bfloat16()
        k = torch.randn(rows, cols, generator=g, device="cuda").bfloat16() if skip else None
        check_backward(dy, out["res"], w, out["rstd"], k, *backward(dy, out["res"], w, out["rstd"], k))


def test_norm_gradients_against_differences():
    """Central differences of sum(c * y) in float64, at the kernel's own inputs."""
    x, _, w = make(3, 40, 9, False, True)
    rstd = forward(x, None, w, q=False)["rstd"]
    c = torch.randn(3, 40, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    dx, dw = backward(c, x, w, rstd)
    X, W, C, h = f64(x), f64(w), f64(c), 1e-5
    loss = lambda X, W: (C * N.rmsnorm(X, None, W, EPS)[2]).sum()   # noqa: E731
    for i, j in ((0, 0), (1, 17), (2, 39)):
        d = np.zeros_like(X)
        d[i, j] = h
        num = (loss(X + d, W) - loss(X - d, W)) / (2 * h)
        assert abs(num - f64(dx)[i, j]) <= U16 * abs(num) + 2e-5      # bf16; differences are good to 1e-8, rstd to 6e-6
    for j in (0, 39):
        d = np.zeros_like(W)
        d[j] = h
        num = (loss(X, W + d) - loss(X, W - d)) / (2 * h)
        assert abs(num - f64(dw)[j]) <= 2e-5 * max(1, abs(num))


def test_norm_backward_in_place_of_no_rows_and_the_same_every_time():
    x, r, w = make(333, 1000, 4)
    out = forward(x, r, w, q=False)
    dy, k = torch.randn_like(x), torch.randn_like(x)
    dx, dw = backward(dy, out["res"], w, out["rstd"], k)
    again = backward(dy, out["res"], w, out["rstd"], k)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
    ws = torch.empty(B.moe_rmsnorm_backward_workspace_bytes(333, 1000), dtype=torch.uint8, device="cuda")
    for which in range(3):                                   # dx over dy, over dres, over s
        bufs = [dy.clone(), k.clone(), out["res"].clone()]
        B.moe_rmsnorm_backward(bufs[0], bufs[2], w, out["rstd"], bufs[which], again[1], ws, dres=bufs[1])
        assert torch.equal(bufs[which], dx) and torch.equal(again[1], dw)
    dw.fill_(7)
    B.moe_rmsnorm_backward(dy[:0], x[:0], w, out["rstd"][:0], dx[:0], dw, None)
    assert (dw == 0).all()


def test_norm_captured_and_on_another_stream():
    x, r, w = make(64, 4096, 5)
    want, dyw = forward(x, r, w), torch.randn_like(x)
    bwd = backward(dyw, want["res"], w, want["rstd"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, q, sc, rs, res = (torch.zeros_like(want[n]) for n in ("y", "q", "scale", "rstd", "res"))
    dx, dw = torch.zeros_like(bwd[0]), torch.zeros_like(bwd[1])
    ws = torch.empty(B.moe_rmsnorm_backward_workspace_bytes(64, 4096), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    xs = x.clone()
    with torch.cuda.graph(graph, stream=side):
        B.moe_rmsnorm(xs, w, EPS, y=y, residual=r, res_out=res, yq=q, scale=sc, rstd=rs)
        B.moe_rmsnorm_backward(dyw, res, w, rs, dx, dw, ws)
    xs.zero_()
    graph.replay()
    xs.copy_(x)
    graph.replay()
    torch.cuda.synchronize()
    for got, name in ((y, "y"), (q, "q"), (sc, "scale"), (rs, "rstd"), (res, "res")):
        assert torch.equal(got, want[name]), name
    assert torch.equal(dx, bwd[0]) and torch.equal(dw, bwd[1])


def test_norm_backward_by_two_threads_at_once():
    """Widths that share a kernel and differ in its shared memory: neither thread takes from the other what its launch needs."""
    import threading
    jobs, errors = [], []
    for cols in (4104, 8192, 6000):
        x, r, w = make(40, cols, cols)
        out, dy, k = forward(x, r, w, q=False), torch.randn_like(x), torch.randn_like(x)
        jobs.append((cols, out, w, dy, k, backward(dy, out["res"], w, out["rstd"], k), torch.empty_like(x),
                     torch.empty(cols, device="cuda"),
                     torch.empty(B.moe_rmsnorm_backward_workspace_bytes(40, cols), dtype=torch.uint8, device="cuda"),
                     torch.cuda.Stream()))
    torch.cuda.synchronize()

    def run(cols, out, w, dy, k, want, dx, dw, ws, stream):
        try:
            for _ in range(400):
                B.moe_rmsnorm_backward(dy, out["res"], w, out["rstd"], dx, dw, ws, dres=k, stream=stream)
            stream.synchronize()
            assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
        except Exception as e:   # noqa: BLE001
            errors.append((cols, e))

    threads = [threading.Thread(target=run, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors


@pytest.mark.parametrize("cols", [512, 1024, 2048, 4096, 8192, 16384])
@pytest.mark.parametrize("res", [False, True])
def test_norm_rows_whose_sum_of_squares_is_not_finite(cols, res):
    """NaN throughout, not zeros that look like a result: a NaN, an infinity, values whose squares or whose sum of squares leave fp32, and a sum with the
    residual that does.  The rows beside them are those of a call without them."""
    x, r, w = make(9, cols, cols, res)
    want = forward(x, r, w)
    bad = torch.tensor([1, 2, 3, 4, 6, 7], device="cuda")
    x[1, 3], x[2, cols - 1], x[3, 0] = float("nan"), float("inf"), -float("inf")
    x[4, 5] = 2e19                               # its square is not finite
    x[6] = 1.8e19                                # each square is, their sum is not
    if res:
        x[7], r[7] = 3e38, 3e38
    else:
        x[7] = -3.3e38
    out = forward(x, r, w)
    good = torch.tensor([0, 5, 8], device="cuda")
    for name, t in out.items():
        assert torch.equal(t[good], want[name][good]), name
    assert torch.isnan(out["y"][bad]).all() and torch.isnan(out["rstd"][bad]).all() and torch.isnan(out["scale"][bad]).all()
    assert np.isnan(e4m3(out["q"][bad])).all()
    if res:
        assert torch.equal(torch.nan_to_num(out["res"], 7.0), torch.nan_to_num((x.float() + r.float()).bfloat16(), 7.0))
    # the backward passes the NaN on, to its own rows of dx and to dw
    g = torch.Generator(device="cuda").manual_seed(1)
    dy = torch.randn(9, cols, generator=g, device="cuda").bfloat16()
    s = out["res"] if res else x
    dx, dw = backward(dy, s, w, out["rstd"])
    assert torch.isnan(dx[bad]).all() and torch.isfinite(dx[good]).all() and torch.isnan(dw).all()


def test_norm_of_large_values_within_range():
    """Squares near the end of fp32, and at its beginning with eps = 0."""
    for cols in (64, 4096, 16384):
        x, r, w = make(40, cols, 2, True, True)
        top = 1.8e19 / (5 * cols) ** 0.5 / 4     # cols squares of about 0.6 top^2 are 2.5e36
        x, r = (x.float() * top / 4).bfloat16(), (r.float() * top / 4).bfloat16()
        check_forward(x, r, w, forward(x, r, w))
    # eps = 0 and squares that vanish: NaN, as for a row of zeros
    tiny = forward(torch.full((1, 256), 1e-25, device="cuda").bfloat16(), None, torch.ones(256, device="cuda"), eps=0.0)
    assert torch.isnan(tiny["y"]).all() and torch.isnan(tiny["scale"]).all() and torch.isnan(tiny["rstd"]).all()


def test_norm_backward_of_the_most_rows():
    """2^31 - 1 rows, the limit: row numbers and the rounding up to whole blocks need more than 32 bits.  Rows of 8 columns, dx over dy."""
    rows, cols = (1 << 31) - 1, 8
    if torch.cuda.mem_get_info()[0] < 100e9:
        pytest.skip("needs 86 GB of device memory")
    s = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    dy = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    rstd = torch.full((rows,), 0.5, device="cuda")
    hot = [0, 7, 4735, 1 << 30, rows - 9, rows - 8, rows - 1]
    for i in hot:
        dy[i, 3] = 2.0
    w, dw = torch.ones(cols, device="cuda"), torch.full((cols,), 7.0, device="cuda")
    ws = torch.empty(B.moe_rmsnorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.moe_rmsnorm_backward(dy, s, w, rstd, dy, dw, ws)
    torch.cuda.synchronize()
    # g = 2 e_3, xhat = 0.5: dx = 0.5 (g - 0.5 * mean(g * 0.5)) = e_3 - 0.03125; dw_3 = 2 * 0.5 per row
    want = torch.full((cols,), -0.03125)
    want[3] += 1
    for i in hot:
        assert torch.equal(dy[i].float().cpu(), want), i
        dy[i] = 0
    assert dw.tolist() == [0, 0, 0, len(hot), 0, 0, 0, 0]
    assert not any(part.any().item() for part in dy.split(1 << 27))
    del s, dy, rstd
    torch.cuda.empty_cache()


# ---- more rows than blocks ---------------------------------------------------------------------------------------------------
def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def varied(rows, cols, seed, std=1.0):
    """Rows whose size differs from one to the next by up to 16 times: a sum that is taken from another row shows."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    size = torch.exp2(4 * torch.rand(rows, 1, generator=g, device="cuda"))
    return (torch.randn(rows, cols, generator=g, device="cuda") * size * std).bfloat16()


# as launched: at most 64 blocks per SM for 1025 to 4096 columns, 16 for the others; a block takes eight rows at once up to 1024 columns, else one
@pytest.mark.parametrize("cols", [64, 640, 1536, 4096, 7168, 10000, 16384])
@pytest.mark.parametrize("res,y,q", [(True, True, True), (False, True, False), (True, False, True), (False, True, True), (True, True, False)])
def test_norm_when_blocks_take_several_rows(cols, res, y, q):
    rows = 2 * sms() * (64 if 1024 < cols <= 4096 else 16) * (8 if cols <= 1024 else 1) + 5
    x, r = varied(rows, cols, cols), varied(rows, cols, cols + 1) if res else None
    w = 1 + 0.3 * torch.randn(cols, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    out = forward(x, r, w, y, q)
    wd = w.double()
    for i in range(0, rows, 4096):
        n = slice(i, min(rows, i + 4096))
        s = x[n].double() + (r[n].double() if res else 0.0)
        rstd = 1 / torch.sqrt(s.square().mean(1) + EPS)
        ref = s * rstd[:, None] * wd
        assert ((out["rstd"][n].double() - rstd).abs() <= CHAIN * U32 * rstd).all()
        if res:
            assert ((out["res"][n].double() - s).abs() <= (U16 + U32) * s.abs()).all()
        err = (CHAIN + 4) * U32 * ref.abs()
        if y:
            assert ((out["y"][n].double() - ref).abs() <= U16 * ref.abs() + (1 + U16) * err).all()
        if q:
            sc = out["scale"][n].double()
            top = ref.abs().amax(1) / 448
            assert ((sc - top).abs() <= (CHAIN + 6) * U32 * top).all()
            got = out["q"][n].view(torch.float8_e4m3fn).double() * sc[:, None]
            assert ((got - ref).abs() <= (2.0 ** -4 + 2.0 ** -18) * ref.abs() + 2.0 ** -10 * sc[:, None]).all()


# rows so that every stage of a block's ring (4 up to 512 and to 4096 columns, 3 to 1024 and to 8192, else 2) is filled at least three times
@pytest.mark.parametrize("cols,rows", [(64, 60001), (640, 45003), (1504, 7500), (1536, 7500), (2880, 7500), (4096, 7500), (5000, 5500), (7168, 5500), (8192, 5500),
                                       (12000, 3800), (16384, 3800)])
@pytest.mark.parametrize("skip", [False, True])
def test_norm_backward_when_the_ring_is_filled_again(cols, rows, skip):
    n = sms()
    assert rows > 3 * (4 if cols <= 512 or 1024 < cols <= 4096 else 3 if cols <= 8192 else 2) * 4 * n * (8 if cols <= 1024 else 1)
    s, dy = varied(rows, cols, cols, 0.5), varied(rows, cols, cols + 1, 0.1)
    k = varied(rows, cols, cols + 2, 0.1) if skip else None
    w = 1 + 0.3 * torch.randn(cols, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    rstd = torch.rsqrt(s.float().square().mean(1) + EPS)
    dx, dw = backward(dy, s, w, rstd, k)
    wd, dw_ref, dw_mag = w.double(), torch.zeros(cols, dtype=torch.float64, device="cuda"), torch.zeros(cols, dtype=torch.float64, device="cuda")
    for i in range(0, rows, 4096):
        m = slice(i, min(rows, i + 4096))
        rv = rstd[m].double()[:, None]
        xhat, a = s[m].double() * rv, dy[m].double()
        g = a * wd
        ref = rv * (g - xhat * (g * xhat).mean(1, keepdim=True)) + (k[m].double() if skip else 0.0)
        mag = rv * (6 * g.abs() + xhat.abs() * (CHAIN + 6) * (g * xhat).abs().mean(1, keepdim=True))   # as in check_backward
        err = U32 * (mag + ref.abs() + (k[m].double().abs() if skip else 0.0))
        assert ((dx[m].double() - ref).abs() <= U16 * ref.abs() + (1 + U16) * err).all()
        dw_ref += (a * xhat).sum(0)
        dw_mag += (a * xhat).abs().sum(0)
    # additions in a row: a block's rows (one block per SM at least), its eight warps, a warp's share of at most 592 blocks, the 32 lanes; 4 for a term
    depth = -(-rows // n) + 8 + -(-592 // 32) + 5 + 4
    assert ((dw.double() - dw_ref).abs() <= depth * U32 * dw_mag).all()
    # over its inputs, and the same bits every time
    again = torch.empty_like(dw)
    ws = torch.empty(B.moe_rmsnorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    for t in (dy, s, k):
        if t is not None:
            kept = t.clone()
            B.moe_rmsnorm_backward(dy, s, w, rstd, t, again, ws, dres=k)
            assert torch.equal(t, dx) and torch.equal(again, dw)
            t.copy_(kept)
