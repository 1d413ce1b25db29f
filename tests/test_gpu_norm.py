"""Layer norm on the GPU against its 64-bit form, within bounds that follow from
fp32 arithmetic (norm_reference.py)."""
import pytest
import torch

import norm_reference as ref

pytestmark = pytest.mark.gpu

from paper_2603_18112_amd import ags, norm  # noqa: E402

F, B = torch.float32, torch.bfloat16
# each kernel's widths at their ends, odd ones, few and many rows
SIZES = [(1, 1), (3, 1), (1, 16), (5, 7), (64, 512), (65, 513), (33, 1000), (33, 1024), (17, 1025), (9, 2048),
         (5, 2049), (1, 4096), (300, 4096), (3, 4097), (2, 8192), (2, 8193), (2, 16384), (3, 16385), (2, 32768),
         (3, 32769), (700, 100), (2500, 520), (6000, 40), (40, 40000)]


def _inputs(rows, cols, dtype, seed=0, offset=0.5):
    gen = torch.Generator().manual_seed(seed * 7919 + rows * 131 + cols)
    x = torch.randn(rows, cols, generator=gen) * torch.exp(0.5 * torch.randn(cols, generator=gen)) + offset
    dy = torch.randn(rows, cols, generator=gen) * 0.01
    if rows > 2:
        x[1], dy[1] = 0.0, 0.0          # a padding row
        x[2] = 3.0                      # a constant one
    w, b = torch.randn(cols, generator=gen) * 0.2 + 1.0, torch.randn(cols, generator=gen)
    return x.to(dtype), dy.to(dtype), w, b


def _within(got, want, tol, what):
    got = got.double().cpu()
    off = (got - want).abs() - tol
    assert torch.isfinite(got).all(), what
    assert (off <= 0).all(), f"{what}: {float(off.max()):.3g} beyond its bound"


def _check_forward(x, w, b, y, saved, eps=1e-5):
    (ry, rm, rr), (ey, em, er) = ref.forward(x.cpu(), w, b, eps, y.dtype)
    _within(y.reshape(ry.shape), ry, ey, "y")
    _within(saved[0], rm, em, "mean")
    _within(saved[1], rr, er, "rstd")


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype,w_dtype", [(F, F), (B, F), (B, B)])
def test_both_passes(rows, cols, dtype, w_dtype):
    x, dy, w, b = _inputs(rows, cols, dtype)
    w, b = w.to(w_dtype), b.to(w_dtype)
    xc, dc, wc, bc = (t.cuda() for t in (x, dy, w, b))
    y, saved = norm.layer_norm(xc, wc, bc, save=True)
    assert y.dtype == dtype and saved.shape == (2, rows)
    _check_forward(x, w, b, y, saved)
    dx, dw, db = norm.layer_norm_backward(dc, xc, saved, wc)
    want, tol = ref.backward(dy, x, saved.cpu(), w, dtype, F)
    for got, r, t, what in zip((dx, dw, db), want, tol, ("dx", "dweight", "dbias")):
        _within(got, r, t, what)
    # each result by itself, bit for bit
    only = norm.layer_norm_backward(dc, xc, saved, wc, need_dw=False, need_db=False)
    assert torch.equal(only[0], dx) and only[1] is None and only[2] is None
    only = norm.layer_norm_backward(dc, xc, saved, wc, need_dx=False, need_db=False)
    assert only[0] is None and torch.equal(only[1], dw) and only[2] is None
    only = norm.layer_norm_backward(dc, xc, saved, wc, need_dx=False, need_dw=False)
    assert torch.equal(only[2], db)
    assert torch.equal(norm.layer_norm(xc, wc, bc), y)


@pytest.mark.parametrize("rows,cols", [(7, 33), (4, 1500), (3, 40000)])
@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (False, True)])
def test_without_weight_or_bias_and_other_output_types(rows, cols, weight, bias):
    x, dy, w, b = _inputs(rows, cols, B, 1)
    w, b = w if weight else None, b if bias else None
    wc, bc = None if w is None else w.cuda(), None if b is None else b.cuda()
    y, saved = norm.layer_norm(x.cuda(), wc, bc, dtype="f32", save=True)
    assert y.dtype == F
    _check_forward(x, w, b, y, saved)
    y = norm.layer_norm(x.float().cuda(), wc, bc, dtype=B)
    assert y.dtype == B
    _check_forward(x.float(), w, b, y, saved)
    dx, dw, db = norm.layer_norm_backward(dy.cuda(), x.cuda(), saved, wc, dw_dtype="bf16")
    want, tol = ref.backward(dy, x, saved.cpu(), w, B, B)
    for got, r, t, what in zip((dx, dw, db), want, tol, ("dx", "dweight", "dbias")):
        _within(got, r, t, what)


@pytest.mark.parametrize("cols", [300, 3000, 20000])
def test_strides_shapes_and_rows_left_alone(cols):
    """A slice of wider rows (odd ones: no alignment), an output gradient that is
    broadcast, results in views of larger buffers, which stay as they were."""
    x, dy, w, b = _inputs(6, cols, B, 2)
    wide = torch.zeros(6, cols + 7, dtype=B).cuda()
    wide[:, 3:3 + cols] = x.cuda()
    xs = wide[:, 3:3 + cols]
    y, saved = norm.layer_norm(xs.view(6, cols) if xs.is_contiguous() else xs, w.cuda(), b.cuda(), save=True)
    _check_forward(x, w, b, y, saved)
    y3 = norm.layer_norm(x.view(2, 3, cols).cuda(), w.cuda(), b.cuda())
    assert y3.shape == (2, 3, cols) and torch.equal(y3.view(6, cols), y)
    yt = norm.layer_norm(x.t().contiguous().cuda().t(), w.cuda(), b.cuda())
    assert torch.equal(yt, y)
    spread = dy[:1].expand(6, cols)
    row = torch.full((2 * cols + 9,), 5.0).cuda()
    dx, dw, db = norm.layer_norm_backward(spread.cuda().expand(6, cols), xs, saved, w.cuda(),
                                          dweight=row[1:1 + cols], dbias=row[1 + cols:1 + 2 * cols])
    want, tol = ref.backward(spread, x, saved.cpu(), w, B, F)
    for got, r, t, what in zip((dx, row[1:1 + cols], row[1 + cols:1 + 2 * cols]), want, tol, ("dx", "dw", "db")):
        _within(got, r, t, what)
    assert (row[:1] == 5).all() and (row[1 + 2 * cols:] == 5).all()
    assert (wide[:, :3] == 0).all() and (wide[:, 3 + cols:] == 0).all()
    # through the C-ABI: rows of y and dx that lie apart
    y2 = torch.full((6, cols + 5), 9.0, dtype=B).cuda()
    s = torch.cuda.current_stream().cuda_stream
    norm.ags_layer_norm(xs.data_ptr(), ags.AGS_BF16, 6, cols, cols + 7, w.cuda().data_ptr(), None, ags.AGS_F32, 1e-5,
                        y2.data_ptr(), ags.AGS_BF16, cols + 5, None, s)
    assert torch.equal(y2[:, :cols], norm.layer_norm(x.cuda(), w.cuda())) and (y2[:, cols:] == 9).all()
    norm.ags_layer_norm_backward(dy.cuda().data_ptr(), cols, xs.data_ptr(), ags.AGS_BF16, 6, cols, cols + 7,
                                 saved.data_ptr(), None, ags.AGS_F32, y2.data_ptr(), cols + 5, None, None,
                                 ags.AGS_F32, stream=s)
    dx = norm.layer_norm_backward(dy.cuda(), x.cuda(), saved, need_dw=False, need_db=False)[0]
    assert torch.equal(y2[:, :cols], dx) and (y2[:, cols:] == 9).all()


@pytest.mark.parametrize("dw_dtype", [F, B])
def test_gradients_added(dw_dtype):
    x, dy, w, b = _inputs(500, 700, B, 3)
    old = torch.randn(2, 700).to(dw_dtype)
    dw, db = (t.clone() for t in old.cuda())
    _, saved = norm.layer_norm(x.cuda(), save=True)
    norm.layer_norm_backward(dy.cuda(), x.cuda(), saved, w.cuda(), dweight=dw, dbias=db, accumulate=True)
    (_, rw, rb), (_, tw, tb) = ref.backward(dy, x, saved.cpu(), w, B, F)
    for got, r, t, o in ((dw, rw, tw, old[0]), (db, rb, tb, old[1])):
        r = r + o.double()
        _within(got, r, t + r.abs() * (ref.U + ref.HALF[dw_dtype]), "added")


def test_empty():
    w = torch.ones(8).cuda()
    y, saved = norm.layer_norm(torch.empty(0, 8).cuda(), w, save=True)
    assert y.shape == (0, 8) and saved.shape == (2, 0)
    dx, dw, db = norm.layer_norm_backward(y, y, saved, w)
    assert dx.shape == (0, 8) and (dw == 0).all() and (db == 0).all()
    dw.fill_(3.0)
    norm.layer_norm_backward(y, y, saved, w, dweight=dw, dbias=db, accumulate=True)
    assert (dw == 3).all()
    assert norm.layer_norm_backward(y, y, saved, w, need_dw=False, need_db=False)[0].shape == (0, 8)
    y, saved = norm.layer_norm(torch.empty(4, 0).cuda(), save=True)
    assert y.shape == (4, 0)
    assert norm.layer_norm_backward(y, y, saved)[1].shape == (0,)


@pytest.mark.parametrize("cols", [200, 5000, 40000])
def test_nonfinite_rows_stay_by_themselves(cols):
    x, dy, w, b = _inputs(4, cols, F, 4)
    good = norm.layer_norm(x.cuda(), w.cuda(), b.cuda(), save=True)
    gx = norm.layer_norm_backward(dy.cuda(), x.cuda(), good[1], w.cuda())[0]
    x[0, 3], x[3, cols - 1] = float("inf"), float("nan")
    y, saved = norm.layer_norm(x.cuda(), w.cuda(), b.cuda(), save=True)
    assert torch.isnan(y[0]).all() and torch.isnan(y[3]).all() and torch.equal(y[1:3], good[0][1:3])
    dx = norm.layer_norm_backward(dy.cuda(), x.cuda(), saved, w.cuda())[0]
    assert torch.isnan(dx[0]).all() and torch.isnan(dx[3]).all() and torch.equal(dx[1:3], gx[1:3])


def test_large_offsets_and_extremes():
    """A mean far above the spread; values whose squares overflow or vanish in
    fp32 are outside what the formula holds in fp32, those here are inside."""
    x, _, w, b = _inputs(8, 777, F, 5, offset=1000.0)
    y, saved = norm.layer_norm(x.cuda(), w.cuda(), b.cuda(), save=True)
    _check_forward(x, w, b, y, saved)
    x = x * 1e12
    y, saved = norm.layer_norm(x.cuda(), w.cuda(), b.cuda(), save=True)
    _check_forward(x, w, b, y, saved)
    x = x * 1e-24
    y, saved = norm.layer_norm(x.cuda(), w.cuda(), b.cuda(), eps=0.0, save=True)
    keep = torch.tensor([0, 1, 3, 4, 5, 6, 7])[2:]       # rows 1 and 2 are constant: 0 / 0
    _check_forward(x[keep], w, b, y[keep], saved[:, keep], eps=0.0)
    assert torch.isnan(y[1]).all()


def test_gradient_against_differences():
    x, _, w, b = _inputs(3, 50, F, 6)
    r = torch.randn(3, 50, dtype=torch.float64, generator=torch.Generator().manual_seed(1))

    def loss(xd, wd, bd):
        return float((ref.forward(xd, wd, bd, 1e-5, F)[0][0] * r).sum())

    y, saved = norm.layer_norm(x.cuda(), w.cuda(), b.cuda(), save=True)
    dx, dw, db = (t.cpu().double() for t in norm.layer_norm_backward(r.float().cuda(), x.cuda(), saved, w.cuda()))
    h = 1e-5
    for t, grad, at in ((x.double(), dx, (0, 7)), (x.double(), dx, (2, 49)), (w.double(), dw, (9,)), (b.double(), db, (11,))):
        up, down = t.clone(), t.clone()
        up[at] += h
        down[at] -= h
        args = [x.double(), w.double(), b.double()]
        i = 0 if t.dim() == 2 else 1 if grad is dw else 2
        args[i] = up
        hi = loss(*args)
        args[i] = down
        # differences: h^2 of a third derivative of order 10, and 64-bit rounding over h
        assert abs((hi - loss(*args)) / (2 * h) - float(grad[at])) < 1e-4 * max(1.0, abs(float(grad[at])))


def test_streams_and_graphs():
    """On another stream than the tensors', and replayed from a graph with eager
    work between the replays."""
    x, dy, w, b = (t.cuda() for t in _inputs(257, 1111, B, 7))
    want = norm.layer_norm(x, w, b, save=True)
    grads = norm.layer_norm_backward(dy, x, want[1], w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = norm.layer_norm(x, w, b, save=True)
        back = norm.layer_norm_backward(dy, x, got[1], w)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and all(torch.equal(p, q) for p, q in zip(back, grads))
    dw, db = torch.zeros(1111).cuda(), torch.zeros(1111).cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, saved = norm.layer_norm(x, w, b, save=True)
        dx, _, _ = norm.layer_norm_backward(dy, x, saved, w, dweight=dw, dbias=db)
    for seed in (8, 9, 10):
        x2, dy2, _, _ = _inputs(257, 1111, B, seed)
        x.copy_(x2)
        dy.copy_(dy2)
        graph.replay()
        torch.cuda.synchronize()
        e, s = norm.layer_norm(x, w, b, save=True)
        g = norm.layer_norm_backward(dy, x, s, w)
        assert torch.equal(y, e) and torch.equal(dx, g[0]) and torch.equal(dw, g[1]) and torch.equal(db, g[2])


def test_offsets_past_32_bits():
    """Rows whose elements lie beyond 2^32 of the buffer, by a stride that leaves
    room between them."""
    cols, stride = 96, 1 << 31
    buf = torch.empty(2 * stride + 2 * cols, dtype=B, device="cuda")
    x = torch.as_strided(buf, (3, cols), (stride, 1))
    x.copy_(_inputs(3, cols, B, 11)[0])
    y, saved = norm.layer_norm(x, save=True)
    _check_forward(x.cpu(), None, None, y, saved)
    dy = torch.ones(3, cols, dtype=B, device="cuda")
    a = norm.layer_norm_backward(dy, x, saved)
    c = norm.layer_norm_backward(dy, x.contiguous(), saved)
    assert all(torch.equal(p, q) for p, q in zip(a, c))


def test_binding_refuses():
    x, w = torch.zeros(4, 8).cuda(), torch.zeros(8).cuda()
    saved = torch.zeros(2, 4).cuda()
    f, g = norm.layer_norm, norm.layer_norm_backward
    for args, kw in (((x, w[:7]), {}), ((x, w, w.bfloat16()), {}), ((x.half(),), {}), ((x, w.cpu()), {}),
                     ((x.requires_grad_(),), {}), ((x.detach(), w), {"dtype": "fp8"}), ((torch.tensor(1.0).cuda(),), {})):
        with pytest.raises(ValueError):
            f(*args, **kw)
    x = x.detach()
    for args, kw in (((x, x, saved[:, :3]), {}), ((x, x, saved.double()), {}), ((x.bfloat16(), x, saved), {}),
                     ((x, x, saved, w), {"accumulate": True}), ((x, x, saved, w), {"dweight": w, "need_dw": False}),
                     ((x, x, saved, w), {"dweight": w[:3]}), ((x, x, saved, w), {"dweight": w.bfloat16()})):
        with pytest.raises(ValueError):
            g(*args, **kw)
    with pytest.raises(ags.AGSError):
        f(x, eps=-1.0)
    with pytest.raises(ags.AGSError):
        g(x, x, saved, w, dweight=w, dbias=x[0])             # dbias over dy
