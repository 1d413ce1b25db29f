"""The 4-bit operators on the GPU against their definition in 64 bits.

Stored values are compared exactly: the format leaves nothing to rounding.
Products of small whole numbers are compared exactly too, their fp32 sums
being exact in any order.  Other products: every one of the k additions may
be off by 2^-23 of the sum of magnitudes (a truncating adder), the result by
its rounding (2^-24, or 2^-8 for bf16).
"""
import numpy as np
import pytest

import mx_reference as ref
from paper_2603_18112_amd import ags, mx

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    yield
    torch.cuda.synchronize()


def rand(rows, cols, dtype="f32", seed=0, spread=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn(rows, cols, device="cuda", generator=gen)
    x *= (torch.randn(rows, cols, device="cuda", generator=gen) * spread).exp()
    return x.to(DT[dtype])


def noise_of(rows, cols, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 77)
    return torch.randint(0, 256, (rows, cols), device="cuda", generator=gen, dtype=torch.uint8)


def f64(t):
    return t.detach().double().cpu().numpy()


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


def check_packed(q, want, exps):
    """Codes, scales and padding of an MX4 against values and exponents."""
    rows, cols = q.shape
    codes, scales = q.codes.cpu().numpy(), q.scales.cpu().numpy()
    v = ref.unpack(codes, scales, rows, cols)
    assert same(v[:, :cols], want)
    if rows:
        scales = ref.scale_rows(scales, rows, cols)
        assert same(scales[:, :exps.shape[1]].astype(np.int64) - 127, exps)
        assert not np.any(v[:, cols:]) or np.isnan(want).any()
        kp = v.shape[1]
        n = np.stack([codes & 15, codes >> 4], axis=-1).reshape(rows, kp)
        assert not n[:, cols:].any()                                  # padding codes are zero
        nb = exps.shape[1]
        assert not scales[:, nb:].any()


SHAPES = [(1, 1), (1, 32), (3, 31), (2, 33), (5, 256), (64, 1000), (257, 255), (300, 129), (33, 2047), (256, 512)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("noisy", [False, True])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_store_and_read_back(rows, cols, dtype, noisy):
    x = rand(rows, cols, dtype, rows + cols, 2.0)
    r = noise_of(rows, cols) if noisy else None
    rn = None if r is None else r.cpu().numpy()
    want, e = ref.store_rows(f64(x), rn)
    want_t, e_t = ref.store_rows(f64(x).T, None if rn is None else rn.T)
    q, qt = mx.quantize(x, noise=r), mx.quantize_t(x, noise=r)
    check_packed(q, want, e)
    check_packed(qt, want_t, e_t)
    b, bt = mx.quantize_both(x, noise=r)
    for one, two in ((q, b), (qt, bt)):
        assert torch.equal(one.codes, two.codes)
        if rows and cols:
            assert same(ref.scale_rows(one.scales.cpu().numpy(), *one.shape),
                        ref.scale_rows(two.scales.cpu().numpy(), *two.shape))
    for dt in ("f32", "bf16"):
        assert same(f64(mx.dequantize(q, dt)), want)
        assert same(f64(mx.dequantize(qt, dt)), want_t)


@pytest.mark.parametrize("noisy", [False, True])
def test_every_bf16_value(noisy):
    """All bf16 patterns, sorted by magnitude so that blocks are alike, then in
    their order (ties, denormals, infinities, NaN)."""
    bits = np.arange(65536, dtype=np.uint16)
    order = np.argsort(bits & 0x7FFF, kind="stable")
    for b in (bits[order], bits):
        x = torch.from_numpy(b.astype(np.int16)).cuda().view(torch.bfloat16).view(64, 1024)
        r = noise_of(64, 1024) if noisy else None
        rn = None if r is None else r.cpu().numpy()
        with np.errstate(invalid="ignore"):
            want, e = ref.store_rows(f64(x), rn)
            want_t, e_t = ref.store_rows(f64(x).T, None if rn is None else rn.T)
        q, qt = mx.quantize_both(x, noise=r)
        check_packed(q, want, e)
        check_packed(qt, want_t, e_t)


@pytest.mark.parametrize("noisy", [False, True])
def test_fp32_edges(noisy):
    """Values one bit beside every threshold, at extreme scales."""
    th = np.array([0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7, 7.9999995], np.float32)
    th = np.concatenate([np.nextafter(th, np.float32(0)), th, np.nextafter(th, np.float32(9))])
    rows = []
    for s in (-149, -130, -128, -127, -126, -100, 0, 60, 120, 125, 126):
        for top in (4.0, 6.0, 7.5):
            if np.log2(top) + s >= 128:
                continue
            y = np.ldexp(th.astype(np.float64), s)
            y = np.where(np.abs(y) <= 3.4028234e38, y, 0.0)
            y = np.minimum(y, np.ldexp(top, s))
            rows.append(np.concatenate([y[:31], [np.ldexp(top, s)], -y[-31:], [0.0]]))
    x = torch.from_numpy(np.array(rows).astype(np.float32)).cuda()
    for seed in range(4 if noisy else 1):
        r = noise_of(*x.shape, seed) if noisy else None
        want, e = ref.store_rows(f64(x), None if r is None else r.cpu().numpy())
        check_packed(mx.quantize(x, noise=r), want, e)
        check_packed(mx.quantize_t(x.t().contiguous(), noise=None if r is None else r.t().contiguous()), want, e)


def test_stochastic_thresholds_in_fp32():
    """A fraction just below and at the byte's threshold: an fp32 sum of the
    fraction and the byte would round up over it."""
    x = torch.zeros(256, 32, device="cuda")
    r = torch.zeros(256, 32, device="cuda", dtype=torch.uint8)
    for i in range(256):
        t = 0.5 * (1.0 - (i + 0.5) / 256.0)
        x[i, 0] = 4.0
        for j, base in enumerate((0.0, 0.5, 1.0, 1.5)):
            x[i, 1 + 3 * j] = base + t
            x[i, 2 + 3 * j] = float(np.nextafter(np.float32(base + t), np.float32(0)))
            x[i, 3 + 3 * j] = float(np.nextafter(np.float32(base + t), np.float32(9)))
        r[i] = i
    want, e = ref.store_rows(f64(x), r.cpu().numpy())
    check_packed(mx.quantize(x, noise=r), want, e)


def test_nan_and_infinity_mark_their_block():
    x = rand(40, 100)
    x[3, 40], x[7, 99], x[8, 0] = float("nan"), float("inf"), float("-inf")
    x[9] = -3.4028234e38                                           # a mask of the lowest value is finite
    with np.errstate(invalid="ignore"):
        want, e = ref.store_rows(f64(x))
        want_t, e_t = ref.store_rows(f64(x).T)
    q, qt = mx.quantize_both(x)
    check_packed(q, want, e)
    check_packed(qt, want_t, e_t)
    back = f64(mx.dequantize(q))
    assert np.isnan(back[3, 32:64]).all() and not np.isnan(back[3, :32]).any()
    assert np.isnan(back[7, 96:]).all() and np.isnan(back[8, :32]).all()
    assert np.isfinite(back[9]).all()
    # a marked block reaches every result of its row, and no other
    w = mx.quantize(rand(17, 100, seed=5))
    y = f64(mx.product(q, w, "f32"))
    assert np.isnan(y[[3, 7, 8]]).all() and not np.isnan(np.delete(y, [3, 7, 8], axis=0)).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_and_misaligned_inputs(dtype):
    base = rand(70, 700, dtype)
    r = noise_of(70, 700)
    for view, rv in ((base[:, 1:400], r[:, 1:400]), (base[3:, 8:264], r[3:, 8:264]), (base[::2, :333], r[::2, :333]),
                     (base[5:6, 7:9], r[5:6, 7:9])):
        for n in (None, rv):
            want, e = ref.store_rows(f64(view), None if n is None else n.cpu().numpy())
            want_t, e_t = ref.store_rows(f64(view).T, None if n is None else n.cpu().numpy().T)
            q, qt = mx.quantize_both(view, noise=n)
            check_packed(q, want, e)
            check_packed(qt, want_t, e_t)
            q, qt = mx.quantize_both(view.t(), noise=None if n is None else n.t())     # a transposed view
            check_packed(q, want_t, e_t)
            check_packed(qt, want, e)


def whole(rows, cols, seed, dtype="f32", pad=0):
    """Values that 4 bits hold exactly: grid values times 1, 2 or 4 by block,
    the largest of every block 4 or 6."""
    rng = np.random.default_rng(seed)
    v = rng.choice([-6, -4, -3, -2, -1, -0.5, 0, 0.5, 1, 1.5, 2, 3, 4, 6], size=(rows, cols))
    b = np.repeat(2.0 ** rng.integers(0, 3, (rows, -(-cols // 32))), 32, axis=1)[:, :cols]
    v[:, ::32] = 4.0
    return v * b


PRODUCTS = [(1, 1, 1), (1, 17, 32), (1, 4096, 640), (2, 100, 257), (7, 33, 96), (13, 1000, 512), (16, 16, 128),
            (17, 65, 1000), (24, 250, 4096), (31, 129, 256), (33, 64, 8192), (63, 65, 300), (64, 512, 2048),
            (100, 96, 800), (128, 128, 128), (129, 257, 511), (250, 1000, 96), (255, 300, 260), (256, 256, 256),
            (257, 511, 1024), (300, 77, 2050), (1000, 40, 64), (520, 1030, 320), (5, 2100, 1300),
            (1801, 1811, 520), (3601, 3587, 300), (3600, 3840, 260)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_products_of_whole_numbers_are_exact(m, n, k):
    a, b = whole(m, k, 1), whole(n, k, 2)
    want = a @ b.T                       # multiples of 1/4 below 2^22: exact in fp32
    assert np.abs(a).sum(axis=1).max() * 24 < 2 ** 22 * 24
    qa, qb = mx.quantize(torch.from_numpy(a).float().cuda()), mx.quantize(torch.from_numpy(b).float().cuda())
    assert same(f64(mx.dequantize(qa)), a) and same(f64(mx.dequantize(qb)), b)
    y = mx.product(qa, qb, "f32")
    assert same(f64(y), want)
    assert same(f64(mx.product(qa, qb, "bf16")), f64(torch.from_numpy(want).float().bfloat16()))
    # into a view, and added to what is there
    out = torch.full((m + 2, n + 5), 9.0, device="cuda")
    view = out[1:m + 1, 2:n + 2]
    mx.product(qa, qb, out=view)
    assert same(f64(view), want)
    mx.product(qa, qb, out=view, accumulate=True)
    assert same(f64(view), 2 * want)
    view.fill_(9.0)
    assert bool((out == 9.0).all())                                # nothing else was written
    out = torch.full((m, n), 3.0, device="cuda", dtype=torch.bfloat16)
    mx.product(qa, qb, out=out, accumulate=True)
    assert same(f64(out), f64(torch.from_numpy(want + 3.0).float().bfloat16()))


def check_close(y, a, b, dtype, k):
    want, mag = a @ b.T, np.abs(a) @ np.abs(b).T
    tol = k * 2.0 ** -23 * mag + ROUND[dtype] * np.abs(want) * 1.01 + 2.0 ** -126
    err = np.abs(f64(y).reshape(want.shape) - want)
    assert np.all(err <= tol), (err.max(), (err - tol).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1, 1, 40), (1, 500, 1000), (3, 64, 4096), (12, 999, 500), (40, 333, 2500),
                                   (130, 260, 700), (300, 600, 1100)])
def test_linear_and_its_gradients(m, n, k, dtype):
    x, w, dy = rand(m, k, dtype, 1), rand(n, k, "f32", 2, 0.0) * 0.1, rand(m, n, dtype, 3) * 1e-3
    r = noise_of(m, n)
    weight = mx.Weight(w)
    vx, vxt = ref.store_rows(f64(x))[0], ref.store_rows(f64(x).T)[0]
    vw, vwt = ref.store_rows(f64(w))[0], ref.store_rows(f64(w).T)[0]
    y = mx.linear(x, weight)
    assert y.dtype == x.dtype
    check_close(y, vx, vw, dtype, k)
    y2, saved = mx.linear(x, weight, dtype="f32", save=True)
    check_close(y2, vx, vw, "f32", k)
    for nz in (None, r):
        rn = None if nz is None else nz.cpu().numpy()
        vd, vdt = ref.store_rows(f64(dy), rn)[0], ref.store_rows(f64(dy).T, None if rn is None else rn.T)[0]
        dx, dw = mx.linear_backward(dy, x, weight, noise=nz)
        check_close(dx, vd, vwt, dtype, n)
        check_close(dw, vdt, vxt, "f32", m)
        dx2, dw2 = mx.linear_backward(dy, saved, weight, noise=nz, dw_dtype="bf16")
        assert torch.equal(dx, dx2) and torch.equal(dw.bfloat16(), dw2)
    none, dw3 = mx.linear_backward(dy, saved, weight, noise=r, need_dx=False)
    assert none is None and torch.equal(dw3, dw)
    acc = torch.ones(n, k, device="cuda")
    mx.linear_backward(dy, saved, weight, noise=r, dw=acc, accumulate=True, need_dx=False)
    assert float((acc - 1 - dw).abs().max()) <= 2.0 ** -22 * (1 + float(dw.abs().max()))


def test_gradients_against_differences():
    """Where 4 bits hold every operand exactly the layer is linear and its
    gradients are the formula's; differences of the loss sum(dy y) agree."""
    m, n, k = 64, 32, 96
    x, w, dy = (torch.from_numpy(whole(*s)).float().cuda() for s in ((m, k, 1), (n, k, 2), (m, n, 3)))
    # exact in the transposed forms too: one scale everywhere, a 4 in every block
    x, w, dy = (t.clamp(-4, 4) for t in (x, w, dy))
    for t in (x, w, dy):
        t[::32], t[:, ::32] = 4.0, 4.0
    W = mx.Weight(w)
    dx, dw = mx.linear_backward(dy, x, W)
    assert same(f64(dx), f64(dy) @ f64(w)) and same(f64(dw), f64(dy).T @ f64(x))

    def loss(x, weight):
        return float((f64(mx.linear(x, weight)) * f64(dy)).sum())

    base = loss(x, W)
    for i, j in ((1, 1), (5, 33), (63, 95)):
        old = float(x[i, j])
        new = 0.0 if old else 1.0                    # both on the grid, no scale changes
        x2 = x.clone()
        x2[i, j] = new
        assert loss(x2, W) - base == (new - old) * float(dx[i, j])
    for i, j in ((1, 1), (31, 50)):
        old = float(w[i, j])
        new = 0.0 if old else 1.0
        w2 = w.clone()
        w2[i, j] = new
        assert loss(x, mx.Weight(w2)) - base == (new - old) * float(dw[i, j])


def test_empty_sizes():
    w = mx.Weight(rand(8, 64))
    assert mx.linear(torch.zeros(0, 64, device="cuda"), w).shape == (0, 8)
    dx, dw = mx.linear_backward(torch.zeros(0, 8, device="cuda"), torch.zeros(0, 64, device="cuda"), w)
    assert dx.shape == (0, 64) and not dw.any()
    assert mx.dequantize(mx.quantize(torch.zeros(5, 0, device="cuda"))).shape == (5, 0)
    zero = mx.linear(torch.zeros(4, 64, device="cuda"), w)
    assert not zero.any()


def test_batched_inputs_and_weight_update():
    x, w = rand(30, 96).view(2, 3, 5, 96), rand(40, 96, seed=4)
    W = mx.Weight(w)
    y = mx.linear(x, W)
    assert y.shape == (2, 3, 5, 40)
    assert torch.equal(y.view(30, 40), mx.linear(x.view(30, 96), W))
    W.update(w * 2)
    assert torch.equal(mx.linear(x, W), 2 * y)
    dx, _ = mx.linear_backward(rand(30, 40, seed=9).view(2, 3, 5, 40), x, W)
    assert dx.shape == x.shape


@pytest.mark.parametrize("m,n,k", [(1, 2000, 3000), (20, 640, 5000), (300, 400, 2000), (64, 64, 9000)])
def test_bitwise_reproducible_and_on_other_streams(m, n, k):
    x, W = rand(m, k, "bf16"), mx.Weight(rand(n, k, seed=1))
    first = mx.linear(x, W, dtype="f32")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        outs = [mx.linear(x, W, dtype="f32") for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)


def test_graph_replay_matches_eager():
    m, n, k = 48, 200, 512
    x, dy = rand(m, k, "bf16"), rand(m, n, "bf16", 2)
    w = rand(n, k, seed=3)
    W = mx.Weight(w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mx.linear(x, W), mx.linear_backward(dy, x, W)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        W.update(w)
        y = mx.linear(x, W)
        dx, dw = mx.linear_backward(dy, x, W)
    for step in range(4):
        x.copy_(rand(m, k, "bf16", 10 + step))
        w.copy_(rand(n, k, "f32", 20 + step))
        graph.replay()
        torch.cuda.synchronize()
        W2 = mx.Weight(w)
        y2 = mx.linear(x, W2)
        dx2, dw2 = mx.linear_backward(dy, x, W2)
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and torch.equal(dx, dx2) and torch.equal(dw, dw2)


def test_large_offsets():
    """Rows whose codes and outputs lie past 2^31 and 2^32 bytes."""
    rows, cols = (1 << 17) + 3, 40_000
    x = torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16)
    x[-2, 39_990:] = 3.0
    x[0, 0] = 1.0
    q = mx.quantize(x)
    w = torch.zeros(5, cols, device="cuda")
    w[2, 39_990:], w[1, 0] = 2.0, 2.0
    y = mx.linear(x, mx.Weight(w, backward=False), dtype="f32")
    assert float(y[-2, 2]) == 60.0 and float(y[0, 1]) == 2.0 and int(torch.count_nonzero(y)) == 2
    back = mx.dequantize(q, "bf16")
    assert torch.equal(back, x)
    del back, y
    wide = mx.product(q, mx.quantize(x[:20_000]), "bf16")      # 131,075 x 20,000: 5 GB
    assert float(wide[0, 0]) == 1.0 and int(torch.count_nonzero(wide)) == 1


def test_refusals():
    w = mx.Weight(rand(8, 64))
    x = rand(4, 64)
    for bad in (lambda: mx.quantize(x.cpu()), lambda: mx.quantize(x.half()), lambda: mx.quantize(x[:, ::2][:, :20]),
                lambda: mx.quantize(x, noise=noise_of(4, 63)), lambda: mx.quantize(x, noise=x),
                lambda: mx.linear(rand(4, 65), w), lambda: mx.linear(x, w, dtype=torch.float16),
                lambda: mx.linear(x, mx.Weight(rand(8, 64), forward=False)),
                lambda: mx.linear_backward(rand(4, 9), x, w), lambda: mx.linear_backward(rand(5, 8), x, w),
                lambda: mx.linear_backward(rand(4, 8), x, mx.Weight(rand(8, 64), backward=False)),
                lambda: mx.product(mx.quantize(x), w.rows, accumulate=True),
                lambda: mx.product(mx.quantize(x), w.rows, out=torch.zeros(4, 9, device="cuda")),
                lambda: mx.dequantize(w.rows, "f16"), lambda: w.update(rand(8, 65)),
                lambda: mx.quantize(x.expand(3, 4, 64)[:, 0].expand(3, 64).as_strided((3, 64), (1, 1)))):
        with pytest.raises(ValueError):
            bad()
    q = mx.quantize(x)
    with pytest.raises(ags.AGSError) as e:
        mx.product(q, mx.quantize(rand(8, 96)))
    assert e.value.status == ags.AGS_E_ARG
    host = torch.zeros(4, 64)
    with pytest.raises(ags.AGSError) as e:
        mx.ags_mx_quantize(host.data_ptr(), ags.AGS_F32, 4, 64, 64, None, 0, q.c, None)
    assert e.value.status == ags.AGS_E_ARG


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(16, 40, 2048), (16, 40, 2049), (17, 40, 1900), (1, 33, 32768), (1, 33, 32769),
                                   (3, 7, 10922), (3, 9, 10923), (15, 23, 31), (16, 8, 1)])
def test_few_rows_either_side_of_one_launch(m, n, k, dtype):
    # and a NaN and an infinity, which reach the results of their blocks alone
    x, w = rand(m, k, dtype, 4), rand(n, k, "f32", 5)
    x[m // 2, k // 3] = float("nan")
    w[n - 1, k - 1] = float("inf")
    y = mx.linear(x, mx.Weight(w, backward=False))
    vx, vw = ref.store_rows(f64(x))[0], ref.store_rows(f64(w))[0]
    bad = np.zeros((m, n), bool)
    bad[m // 2], bad[:, n - 1] = True, True
    got = f64(y)
    assert np.array_equal(np.isnan(got), bad)
    vx[m // 2], vw[n - 1] = 0.0, 0.0
    check_close(torch.from_numpy(np.where(bad, 0.0, got)), vx, vw, dtype, k)


@pytest.mark.parametrize("m,n,k", [
    (9, 8200, 700), (16, 8193, 1030),                                     # few rows in tiles
    (70, 90, 257), (70, 90, 600), (70, 90, 1100), (40, 200, 30000),       # 2, 3 and 5 stages, parts
    (100, 17000, 300), (520, 4001, 515),                                  # more small tiles than fit at once
    (600, 5000, 1500), (2100, 2130, 800)])                                # the middle ones, fitting and not
def test_products_ahead_of_memory(m, n, k):
    test_products_of_whole_numbers_are_exact(m, n, k)


@pytest.mark.parametrize("shape", [(2, 3, 0), (0,), (0, 3, 0), (0, 2, 64), (64,)])
def test_inputs_of_one_or_many_axes_with_empty_ones(shape):
    n, k = 40, shape[-1]
    W = mx.Weight(torch.ones(n, k, device="cuda"))
    y, saved = mx.linear(torch.ones(shape, device="cuda"), W, save=True)
    assert torch.equal(y, mx.linear(torch.ones(shape, device="cuda"), W))
    assert y.shape == (*shape[:-1], n) and bool((y == k).all())
    dx, dw = mx.linear_backward(torch.ones_like(y), saved, W)
    rows = y.numel() // n
    assert dx.shape == shape and dw.shape == (n, k)
    assert bool((dx == n).all()) and bool((dw == rows).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (5, 33, 700), (20, 640, 5000), (130, 64, 9000), (300, 700, 20), (17, 257, 4100)])
def test_training_calls_are_the_separate_ones(m, n, k, dtype):
    x, dy, r = rand(m, k, dtype, 1), rand(m, n, dtype, 2), noise_of(m, n)
    W = mx.Weight(rand(n, k, "f32", 3))
    q, qt = mx.quantize_both(x)
    y, saved = mx.linear(x, W, save=True)
    assert saved.shape == (k, m) and torch.equal(saved.codes, qt.codes)
    assert torch.equal(mx.dequantize(saved), mx.dequantize(qt))
    assert torch.equal(y, mx.product(q, W.rows, dtype))
    for noise in (None, r):
        d, dt = mx.quantize_both(dy, noise=noise)
        dx, dw = mx.linear_backward(dy, saved, W, noise=noise)
        assert dx.dtype is DT[dtype] and torch.equal(dx, mx.product(d, W.cols, dtype))
        assert torch.equal(dw, mx.product(dt, qt, "f32"))
        row = torch.full((2 * n * k + 7,), 2.0, device="cuda", dtype=DT[dtype])
        none, view = mx.linear_backward(dy, saved, W, noise=noise, dw=row[5:5 + n * k].view(n, k), need_dx=False,
                                        accumulate=True)
        want = torch.full((n, k), 2.0, device="cuda", dtype=DT[dtype])
        assert none is None and torch.equal(view, mx.product(dt, qt, out=want, accumulate=True))
        assert bool((row[:5] == 2.0).all()) and bool((row[5 + n * k:] == 2.0).all())


@pytest.mark.parametrize("m,n,k", [(40, 200, 30000), (70, 90, 1100), (3, 65, 300)])
def test_training_calls_stay_inside_their_workspaces(m, n, k):
    x, dy, W = rand(m, k), rand(m, n, seed=1), mx.Weight(rand(n, k, seed=2))
    y, saved = torch.empty(m, n, device="cuda"), mx.MX4(k, m)
    dx, dw = torch.empty(m, k, device="cuda"), torch.empty(n, k, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    for need, call in (
            (mx.ags_mx_linear_save_workspace(m, n, k),
             lambda p, b: mx.ags_mx_linear_save(x.data_ptr(), ags.AGS_F32, m, k, W.rows.c, y.data_ptr(), ags.AGS_F32, n,
                                                saved.c, p, b, s)),
            (mx.ags_mx_linear_backward_workspace(m, n, k, 1),
             lambda p, b: mx.ags_mx_linear_backward(dy.data_ptr(), ags.AGS_F32, m, n, n, None, 0, saved.c, W.cols.c,
                                                    dx.data_ptr(), k, dw.data_ptr(), ags.AGS_F32, k, 0, p, b, s))):
        ws = torch.full((need + 8192,), 0xA5, device="cuda", dtype=torch.uint8)
        call(ws.data_ptr() + 4096, need)
        assert bool((ws[:4096] == 0xA5).all()) and bool((ws[4096 + need:] == 0xA5).all())
    y2, saved2 = mx.linear(x, W, save=True)
    dx2, dw2 = mx.linear_backward(dy, saved2, W)
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and torch.equal(dw, dw2)


def test_inputs_without_axes_are_refused():
    w, one = mx.Weight(rand(8, 64)), torch.ones((), device="cuda")
    for bad in (lambda: mx.linear(one, w), lambda: mx.linear_backward(one, rand(1, 64), w),
                lambda: mx.linear(rand(4, 64).cpu(), w), lambda: mx.quantize(one),
                lambda: mx.linear_backward(rand(4, 8), rand(4, 64), w, accumulate=True),
                lambda: mx.linear_backward(rand(4, 8), rand(4, 64), w, dw=torch.zeros(8, 63, device="cuda")),
                lambda: mx.linear_backward(rand(4, 8), rand(4, 64), w, noise=noise_of(4, 7))):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("m,n,k", [(203, 153, 19645), (45, 7, 9001), (17, 1, 20000), (37, 3, 12345), (35, 66, 9000),
                                   (496, 385, 9000), (33, 2, 8300), (130, 131, 9100), (23, 692, 13000)])
def test_parts_joined_over_rows_of_any_length(m, n, k):
    if (m, n) != (496, 385):
        assert mx.ags_mx_product_workspace(m, n, k) > 0            # in parts
    test_products_of_whole_numbers_are_exact(m, n, k)


def test_an_input_that_requires_a_gradient_is_refused():
    w, x = mx.Weight(rand(8, 64)), rand(4, 64).requires_grad_()
    for save in (False, True):
        with pytest.raises(ValueError, match="gradient"):     # y would lose it without a word
            mx.linear(x, w, save=save)
    with torch.no_grad():
        y, saved = mx.linear(x, w, save=True)
    assert torch.equal(y, mx.linear(x.detach(), w))

    class Linear(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            y, ctx.saved = mx.linear(x, w, save=True)
            return y

        @staticmethod
        def backward(ctx, dy):
            return mx.linear_backward(dy, ctx.saved, w)[0]

    dy = rand(4, 8, seed=1)
    Linear.apply(x).backward(dy)
    assert torch.equal(x.grad, mx.linear_backward(dy, saved, w)[0])
    # gradients asked for by name, and weights that are parameters
    assert torch.equal(mx.linear_backward(dy, x, w)[0], x.grad)
    p = torch.nn.Parameter(rand(8, 64))
    mx.Weight(p).update(p)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m", [1, 6, 60])
def test_layers_take_inputs_of_any_strides(m, dtype):
    n, k = 40, 96
    x, dy, r, W = rand(m, k, dtype, 1), rand(m, n, dtype, 2), noise_of(m, n), mx.Weight(rand(n, k, seed=3))

    def check(x, dy, r):
        y, saved = mx.linear(x.contiguous(), W, save=True)
        dx, dw = mx.linear_backward(dy.contiguous(), saved, W, noise=None if r is None else r.contiguous())
        y2, saved2 = mx.linear(x, W, save=True)
        assert torch.equal(y, y2) and torch.equal(mx.dequantize(saved), mx.dequantize(saved2))
        assert torch.equal(mx.linear(x, W), mx.linear(x.contiguous(), W))
        for form in (x, saved2):
            dx2, dw2 = mx.linear_backward(dy, form, W, noise=r)
            assert torch.equal(dx, dx2) and torch.equal(dw, dw2)

    for other in (lambda t: t.t().contiguous().t(), lambda t: t.repeat_interleave(2, 1)[:, ::2],
                  lambda t: torch.cat([t, t], 1)[:, :t.shape[1]]):
        check(other(x), other(dy), None)
        check(other(x), other(dy), other(r))
    one = torch.ones((), device="cuda", dtype=DT[dtype])
    check(x[:1].expand(m, k), one.expand(m, n), r[:1].expand(m, n))       # a broadcast gradient, as of a sum
    if m % 6 == 0:
        a, b, c = (t.view(2, 3, m // 6, -1).transpose(0, 2) for t in (x, dy, r))
        check(a, b, c)
        check(a[..., ::2].repeat_interleave(2, -1), b, c)


def test_results_of_rows_past_4_gib():
    """Output rows whose bytes lie past 2^31 and 2^32, over a filled buffer."""
    m, n, k = (1 << 17) + 3, 20_000, 300
    a, b = torch.zeros(m, k, device="cuda"), torch.zeros(n, k, device="cuda")
    rows, cols = [0, 60_000, m - 130, m - 2, m - 1], [0, 9_999, n - 1]
    for i, r in enumerate(rows):
        a[r, 7], a[r, 299] = (1.0, 2.0, 3.0, 4.0, 6.0)[i], 1.0
    for j, c in enumerate(cols):
        b[c, 7] = (1.0, -2.0, 4.0)[j]
    out = torch.full((m, n), 9.0, device="cuda", dtype=torch.bfloat16)
    for accumulate in (False, True):
        mx.product(mx.quantize(a), mx.quantize(b), out=out, accumulate=accumulate)
        want = (2 if accumulate else 1) * a[rows][:, 7:8] * b[cols][:, 7]
        assert torch.equal(out[rows][:, cols].float(), want)
        assert int(torch.count_nonzero(out)) == len(rows) * len(cols)


@pytest.mark.parametrize("m,n,k,dtype", [(1, 500, 4096, "bf16"), (40, 200, 30000, "f32"), (23, 692, 13000, "bf16"),
                                         (300, 700, 1000, "f32"), (12, 96, 5000, "f32")])
def test_graph_replays_of_training_and_tokens(m, n, k, dtype):
    # one launch for tokens, tiles in parts with the launch that joins them, and
    # the training calls, replayed between eager calls of the same layer
    x, dy, r = rand(m, k, dtype), rand(m, n, dtype, 2), noise_of(m, n)
    W = mx.Weight(rand(n, k, seed=3))
    acc = torch.zeros(n, k, device="cuda")

    def calls():
        y0 = mx.linear(x, W)
        y, saved = mx.linear(x, W, save=True)
        dx, dw = mx.linear_backward(dy, saved, W, noise=r)
        mx.linear_backward(dy, saved, W, noise=r, dw=acc, accumulate=True, need_dx=False)
        return y0, y, dx, dw

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = calls()
    for step in range(4):
        x.copy_(rand(m, k, dtype, 10 + step))
        dy.copy_(rand(m, n, dtype, 20 + step))
        r.copy_(noise_of(m, n, step))
        acc.fill_(step)
        graph.replay()
        torch.cuda.synchronize()
        replayed, there = [t.clone() for t in got], acc.clone()
        acc.fill_(step)
        want = calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, want)) and torch.equal(there, acc)
