"""Layer norm, routing, the experts' rows and the softmax loss compiled for the CPU (tests/cpu_emulation): values against 64 bits through the
C ABI, and every refusal of an argument.  Buffers sit between guards that nothing may touch."""
import ctypes
import math
import os
import sys

import pytest
import torch

import top_ref as ref
from test_dense_emulation import BUILD_DIR, DT, Guarded, emu_build, place, ptr

pytestmark = pytest.mark.skipif(not emu_build.available(), reason="host clang++ of the ROCm toolchain not found")
PIECES = dict(tt_loss=["-DTT_LOSS_ROOM=40000", "-DTT_LOSS_CUT=64", "-DTT_LOSS_COPY_ROWS=100"], tt_loss_narrow=["-DTT_LOSS_NARROW=0"])  # several pieces of the classes, short rows among them
VARIANTS = {"as it is": ("top", {}), "pieces, large tiles": ("top_large", dict(PIECES, tt_gemm=["-DTT_GEMM_LARGE_TILES=1"])),
            "pieces, direct tiles": ("top_direct", dict(PIECES, tt_gemm_direct=["-DTT_GEMM_DIRECT_TILES=1", "-DTT_GEMM_DIRECT_LEAST=0"]))}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def load(tag):
    from paper_2507_14668_amd import binding
    lib = ctypes.CDLL(emu_build.build_dense(BUILD_DIR, *VARIANTS[tag], top=True))
    real = binding.load_library()
    for name in binding.EXPORTS:
        if hasattr(lib, name) and any(name.startswith("tt_" + s) for s in ("layer", "route", "expert", "cross")):
            getattr(lib, name).restype, getattr(lib, name).argtypes = getattr(real, name).restype, getattr(real, name).argtypes
    return lib


@pytest.fixture(scope="module")
def lib():
    return load("as it is")


@pytest.fixture(scope="module", params=VARIANTS)
def loss_lib(request):
    return load(request.param)


def randn(gen, *s, std=1.0, dtype=F32):
    return (torch.randn(*s, generator=gen) * std).to(dtype)


def intact(*gs):
    assert all(g is None or g.intact() for g in gs)


# ---- layer norm
@pytest.mark.parametrize("n", [3, 100, 700, 2500, 4096, 9000])
def test_layer_norm_of_rows_far_from_zero(lib, n):
    """Rows of equal values give the bias, whatever eps is above zero; rows around 1000 and 3e5 what 64 bits give, as far as a mean of fp32 allows.  With
    chains of at most 46 additions (32 in a thread, 14 across) the first mean is off by a = 46 u |mean| at most, in deviations d; the mean of what it leaves
    by 46 u (1 + d), and u |mean| when it is added; the squares by 49 u (1 + d^2), what is taken off them by 92 u d (1 + d), half of both in the root;
    three roundings more in y, one with the bias."""
    from paper_2507_14668_amd import binding
    gen = torch.Generator().manual_seed(n)
    x = torch.stack([torch.full((n,), 1000.1), torch.full((n,), -0.1), 1000 + torch.randn(n, generator=gen), 3e5 + torch.randn(n, generator=gen)])
    bias, out, stats = torch.randn(n, generator=gen), Guarded((4, n), F32), Guarded((4, 2), F32)
    gx, gb = place(x), place(bias)
    op = binding.CNorm(DT[F32], n, 4, eps=1e-12)
    assert lib.tt_layer_norm_forward(ctypes.byref(op), gx.ptr, None, gb.ptr, out.ptr, stats.ptr, None) == 0
    assert torch.equal(out.t[:2], bias.expand(2, n))
    d = x[2:].double()
    y = (d - d.mean(1, keepdim=True)) / torch.sqrt(d.var(1, unbiased=False, keepdim=True) + 1e-12)
    mean, s, u = d.mean(1, keepdim=True), d.std(1, unbiased=False, keepdim=True), 2.0 ** -24
    a = 46 * u * mean / s
    most = u * (mean / s + 46 * (1 + a) + y.abs() * (4 + 24.5 * (1 + a * a) + 46 * a * (1 + a)) + (y + bias).abs())
    off = (out.t[2:].double() - (y + bias)).abs() - most
    assert float(off.max()) <= 0
    assert bool(((stats.t[2:, :1] - mean).abs() <= u * (mean + 46 * s * (1 + a))).all())
    intact(gx, gb, out, stats)


@pytest.mark.parametrize("rows,n,dtype,affine,pad,shift", [
    (1, 1, F32, True, 0, 0), (3, 7, BF16, True, 1, 1), (5, 64, F32, True, 0, 0), (70, 128, F32, True, 0, 0), (19, 130, F16, True, 3, 1),
    (9, 128, BF16, False, 0, 0), (6, 256, BF16, True, 8, 0), (4, 300, F32, True, 0, 3), (3, 1025, F32, True, 0, 0), (3, 2047, BF16, True, 5, 1),
    (2, 2050, F32, True, 0, 0), (2, 4100, F16, True, 0, 0), (2, 8200, BF16, True, 0, 0), (2, 8200, F32, True, 1, 0), (2, 16400, BF16, True, 0, 1),
    (600, 24, F32, True, 0, 0), (0, 16, F32, True, 0, 0)])
def test_layer_norm(lib, rows, n, dtype, affine, pad, shift):
    from paper_2507_14668_amd import binding
    gen = torch.Generator().manual_seed(rows * 7 + n)
    x, grad = (randn(gen, rows, n, std=2) + randn(gen, rows, 1)).to(dtype), randn(gen, rows, n, dtype=dtype)
    w, b = (randn(gen, n, dtype=dtype), randn(gen, n, dtype=dtype)) if affine else (None, None)
    gx, gg, gw, gb = place(x, n + pad, shift), place(grad, n + pad, shift), place(w, None, shift), place(b, None, shift)
    out, dx = Guarded((rows, n), dtype, n + pad, offset=shift), Guarded((rows, n), dtype, n + pad, offset=shift)
    dw, db, stats = Guarded((1, n), dtype, offset=shift), Guarded((1, n), dtype, offset=shift), Guarded((max(rows, 1), 2), F32)
    op = binding.CNorm(DT[dtype], n, rows, n + pad, n + pad, n + pad, n + pad, 1e-5)
    want = ref.norm64(x, w, b, 1e-5, grad)
    assert lib.tt_layer_norm_forward(ctypes.byref(op), gx.ptr, ptr(gw), ptr(gb), out.ptr, stats.ptr, None) == 0
    ws = Guarded((1, max(1, lib.tt_layer_norm_workspace_bytes(ctypes.byref(op)))), torch.uint8)
    assert lib.tt_layer_norm_backward(ctypes.byref(op), gx.ptr, ptr(gw), stats.ptr, gg.ptr, dx.ptr, dw.ptr, db.ptr, ws.ptr, ws.cols, None) == 0
    if rows:
        ref.check(out.t, *want["out"], "out")
        ref.check(dx.t, *want["dx"], "dx")
        ref.check(dw.t[0], *want["dweight"], "dweight")
        ref.check(db.t[0], *want["dbias"], "dbias")
        alone = Guarded((1, n), dtype)
        assert lib.tt_layer_norm_backward(ctypes.byref(op), gx.ptr, ptr(gw), stats.ptr, gg.ptr, None, alone.ptr, None, ws.ptr, ws.cols, None) == 0
        assert torch.equal(alone.t, dw.t)
        alone = Guarded((rows, n), dtype, n + pad)
        assert lib.tt_layer_norm_backward(ctypes.byref(op), gx.ptr, ptr(gw), stats.ptr, gg.ptr, alone.ptr, None, None, None, 0, None) == 0
        assert torch.equal(alone.t, dx.t)
        intact(alone)
    else:
        assert not dw.t.any() and not db.t.any()
    intact(gx, gg, gw, gb, out, dx, dw, db, stats, ws)


def test_layer_norm_special_rows(lib):
    """Rows of equal values, infinities, NaN, numbers at the type's ends: each in its own row only."""
    from paper_2507_14668_amd import binding
    n = 40
    x = torch.randn(6, n, generator=torch.Generator().manual_seed(0))
    x[1], x[2, 3], x[3, 5], x[4] = 7.0, math.inf, math.nan, 0.0
    out, op = torch.empty_like(x), binding.CNorm(0, n, 6, eps=1e-5)
    assert lib.tt_layer_norm_forward(ctypes.byref(op), x.data_ptr(), None, None, out.data_ptr(), None, None) == 0
    good = torch.tensor([0, 1, 4, 5])
    want = ref.norm64(x[good], eps=1e-5)
    ref.check(out[good], *want["out"], "out")
    assert not out[1].any() and not out[4].any()
    assert out[3].isnan().all() and out[2].isnan().any()


def far_rows(n, gen):
    """(name, row of n, eps): rows whose sums, squares or differences leave what fp32 holds, at either end."""
    f = lambda size: torch.randn(n, generator=gen) * size
    sign = torch.where(torch.arange(n) % 2 == 0, 1.0, -1.0)
    one = torch.full((n,), -3e38)
    one[0] = 3e38
    return [("sum", 1e38 + f(1e36), 1e-5), ("squares", 1e20 * sign, 1e-5), ("ends", 3.3e38 * sign, 1e-5), ("one", one, 1e-5), ("random", f(1e30), 1e-5), ("large", f(3e37), 0.0),
            ("small", 1e-25 * sign, 0.0), ("smaller", f(1e-30), 0.0), ("beside eps", f(1e-19), 1e-38), ("mixed", f(1.0) * 10.0 ** (60 * torch.rand(n, generator=gen) - 25), 1e-5),
            ("near", 1e30 + f(1e24), 1e30), ("ordinary", f(1.0), 0.0)]


def stats_loss(want, rstd):
    """An rstd below 2^-126 has fewer bits in the statistics: off by up to 2^-150."""
    return want.abs() * (2.0 ** -150 / rstd)


@pytest.mark.parametrize("n,dtype", [(2, F32), (8, F32), (100, F32), (40, BF16), (200, BF16), (300, F32), (1000, F32), (3000, F32), (5000, BF16), (6000, F32), (9000, F32), (17000, BF16)])
def test_layer_norm_of_any_size(lib, n, dtype):
    """The norm and its gradients of rows near either end of the range, each between ordinary rows, which have the bits that they have alone."""
    from paper_2507_14668_amd import binding
    gen = torch.Generator().manual_seed(n)
    w, b, grad, plain = randn(gen, n, dtype=dtype), randn(gen, n, dtype=dtype), randn(gen, 3, n, dtype=dtype), randn(gen, 2, n, dtype=dtype)

    def run(x, grad, eps):
        rows = x.shape[0]
        out, dx, dw, db, stats = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(w), torch.empty(rows, 2)
        op = binding.CNorm(DT[dtype], n, rows, eps=eps)
        ws = Guarded((1, lib.tt_layer_norm_workspace_bytes(ctypes.byref(op))), torch.uint8)
        assert lib.tt_layer_norm_forward(ctypes.byref(op), x.data_ptr(), w.data_ptr(), b.data_ptr(), out.data_ptr(), stats.data_ptr(), None) == 0
        assert lib.tt_layer_norm_backward(ctypes.byref(op), x.data_ptr(), w.data_ptr(), stats.data_ptr(), grad.data_ptr(), dx.data_ptr(), dw.data_ptr(), db.data_ptr(), ws.ptr,
                                          ws.cols, None) == 0
        return out, dx, dw, stats
    long = n > 4000  # (seconds a row here: some of them)
    for name, row, eps in far_rows(n, gen)[::4 if long else 1]:
        eps = ctypes.c_float(eps).value
        x = torch.stack([plain[0], row.to(dtype), plain[1]])
        out, dx, dw, stats = run(x, grad, eps)
        want = ref.norm64(x, w, b, eps, grad)
        ref.check(out, *want["out"], name + " out")
        d = x.double() - x.double().mean(1, keepdim=True)
        rstd = 1 / ((d * d).mean(1, keepdim=True) + eps).sqrt()
        ref.check(dx, want["dx"][0], want["dx"][1] + stats_loss(want["dx"][0], rstd), name + " dx")
        ref.check(dw, want["dweight"][0], want["dweight"][1] + stats_loss((grad.double() * d * rstd).abs().sum(0), rstd.min()), name + " dweight")
        alone = run(x[:1], grad[:1], eps)
        assert torch.equal(out[0], alone[0][0]) and torch.equal(dx[0], alone[1][0]) and torch.equal(stats[0], alone[3][0]), name
    for value in (1e38, -3.3e38, 1e20, 1e-30, 2.0 ** -149 if dtype == F32 else 2.0 ** -133)[::4 if long else 1]:  # equal values: the bias, whatever eps
        for eps in (1e-5,) if long else (1e-5, 1e-20, 1e-38):
            x = torch.full((2, n), value).to(dtype)
            out, dx, dw, _ = run(x, grad[:2], eps)
            assert torch.equal(out, b.expand(2, n)) and not dw.any(), (value, eps)
            h = grad[:2].double() * w.double()
            want = (h - h.mean(1, keepdim=True)) * ctypes.c_float(eps).value ** -0.5
            size = (h.abs() + h.abs().mean(1, keepdim=True)) * ctypes.c_float(eps).value ** -0.5
            ref.check(dx, want, (64 + n // 256 + 12) * ref.U * size + ref.rounding(want, dtype), "dx %g" % value)


def test_layer_norm_refusals(lib):
    from paper_2507_14668_amd import binding
    x, out, st, ws = torch.zeros(4, 8), torch.zeros(4, 8), torch.zeros(4, 2), torch.zeros(1 << 16, dtype=torch.uint8)
    w = torch.zeros(8)
    at = ws.data_ptr() + -ws.data_ptr() % 256

    def forward(x=x.data_ptr(), w=w.data_ptr(), b=None, out=out.data_ptr(), stats=None, **kw):
        op = binding.CNorm(0, 8, 4, eps=1e-5)
        for k, v in kw.items():
            setattr(op, k, v)
        return lib.tt_layer_norm_forward(ctypes.byref(op), x, w, b, out, stats, None)
    assert forward() == 0
    for bad in (dict(x=None), dict(out=None), dict(out=x.data_ptr()), dict(out=w.data_ptr()), dict(x=x.data_ptr() + 2), dict(dtype=3), dict(dtype=-1), dict(rows=-1),
                dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(stats=out.data_ptr()), dict(stats=x.data_ptr())):
        assert forward(**bad) == binding.TT_ERR_INVALID_ARG, bad
    for bad in (dict(dim=0), dict(dim=(1 << 20) + 1), dict(rows=2 ** 31 - 1), dict(ld_x=7), dict(ld_out=7), dict(ld_out=1 << 41)):
        assert forward(**bad) == binding.TT_ERR_SHAPE, bad
    assert lib.tt_layer_norm_forward(None, None, None, None, None, None, None) == binding.TT_ERR_INVALID_ARG
    dx, dw = torch.zeros(4, 8), torch.zeros(8)

    def backward(x=x.data_ptr(), stats=st.data_ptr(), g=out.data_ptr(), dx=dx.data_ptr(), dw=dw.data_ptr(), db=None, ws=at, size=4096):
        op = binding.CNorm(0, 8, 4, eps=1e-5)
        return lib.tt_layer_norm_backward(ctypes.byref(op), x, w.data_ptr(), stats, g, dx, dw, db, ws, size, None)
    assert backward() == 0
    for bad in (dict(x=None), dict(stats=None), dict(g=None), dict(dx=out.data_ptr()), dict(dw=dx.data_ptr()), dict(db=dw.data_ptr()), dict(dw=st.data_ptr())):
        assert backward(**bad) == binding.TT_ERR_INVALID_ARG, bad
    for bad in (dict(ws=None), dict(ws=at + 16), dict(size=8)):
        assert backward(**bad) == binding.TT_ERR_WORKSPACE, bad


# ---- routing
ROUTES = [
    # rows, experts, k, dtype, scores, bias, groups, top, renorm, scale, pad
    (1, 1, 1, F32, "softmax", False, 1, 1, True, 1.0, 0),
    (9, 5, 5, F32, "softmax", False, 1, 1, False, 1.0, 0),
    (33, 26, 3, BF16, "softmax", True, 1, 1, False, 1.0, 3),
    (17, 64, 2, F32, "sigmoid", True, 1, 1, True, 2.5, 0),
    (12, 65, 4, F16, "softmax", False, 1, 1, True, 1.0, 1),
    (10, 128, 8, BF16, "sigmoid", False, 4, 2, True, 1.0, 0),
    (14, 256, 8, F32, "sigmoid", True, 8, 4, True, 2.5, 0),
    (8, 300, 64, F32, "softmax", True, 1, 1, True, 1.0, 0),
    (9, 36, 4, F32, "softmax", True, 4, 1, False, 1.0, 0),
    (6, 64, 3, F32, "softmax", True, 64, 5, True, 1.0, 0),     # groups of one
    (5, 1024, 7, BF16, "sigmoid", True, 2, 1, False, 1.0, 0),
    (7, 51, 6, F32, "softmax", True, 3, 3, True, 1.0, 0),      # all groups stay
    (11, 264, 2, F16, "sigmoid", True, 33, 2, True, 1.0, 0),   # more groups than half a wavefront
]


def routed(gen, rows, num, dtype, masked=True):
    z = randn(gen, rows, num, std=1.5) + randn(gen, num, std=0.5)
    if masked and rows > 4:
        z[torch.rand(rows, num, generator=gen) < 0.2] = -math.inf
        z[1] = -math.inf                       # padding
        z[2, 1:] = -math.inf                   # one expert is left
        z[3] = 0.25                            # all the same
    return z.to(dtype)


@pytest.mark.parametrize("rows,num,k,dtype,scores,biased,groups,top,renorm,scale,pad", ROUTES)
def test_route(lib, rows, num, k, dtype, scores, biased, groups, top, renorm, scale, pad):
    from paper_2507_14668_amd import binding
    gen = torch.Generator().manual_seed(num + rows)
    z = routed(gen, rows, num, dtype)
    bias = torch.randint(-50, 51, (num,), generator=gen).float() * 1e-3 if biased else None
    if biased and num > 8:
        bias[4] = -math.inf
    how = dict(scores=scores, renormalize=renorm, scale=scale)
    want_w, want_e = ref.route64(z, k, bias, groups=groups, top_groups=top, **how)
    op = binding.CRoute(DT[dtype], binding.SCORES[scores], rows, num, k, groups, top, int(renorm), scale, num + pad, num + pad)
    gz, gb = place(z, num + pad), place(bias[None] if biased else None)
    e, w = Guarded((rows, k), torch.int64), Guarded((rows, k), F32)
    assert lib.tt_route_forward(ctypes.byref(op), gz.ptr, ptr(gb), e.ptr, w.ptr, None) == 0
    assert torch.equal(e.t, want_e)
    ref.check(w.t, want_w, ref.weights_tol(want_w), "weights")
    g = randn(gen, rows, k)
    gg, dz = place(g), Guarded((rows, num), dtype, num + pad)
    assert lib.tt_route_backward(ctypes.byref(op), gz.ptr, e.ptr, gg.ptr, dz.ptr, None) == 0
    ref.check(dz.t, *ref.route_backward64(z, e.t, g, **how), "dlogits")
    intact(gz, gb, e, w, gg, dz)


def test_route_specials(lib):
    """Ties to the lowest number, NaN first and seen, +infinity, scores that underflow, scores that differ in their last bits."""
    from paper_2507_14668_amd import binding
    z = torch.zeros(6, 8)
    z[1, 5] = math.nan
    z[2, 5] = math.inf
    z[3] = torch.tensor([0.0, -1e4, -1e4, -1e4, -math.inf, -1e4, -1e4, -1e4])
    z[4] = torch.tensor([1.0, 1.0 + 2.0 ** -23, 1.0, 1.0 + 2.0 ** -23, 0, 0, 0, 0])
    z[5, 2], z[5, 6] = math.nan, 3.0
    bias = torch.zeros(8)
    for scores in ("softmax", "sigmoid"):
        op = binding.CRoute(0, binding.SCORES[scores], 6, 8, 3, 1, 1, 0, 1.0)
        e, w = torch.empty(6, 3, dtype=torch.int64), torch.empty(6, 3)
        assert lib.tt_route_forward(ctypes.byref(op), z.data_ptr(), bias.data_ptr(), e.data_ptr(), w.data_ptr(), None) == 0
        assert e[0].tolist() == [0, 1, 2] and e[4].tolist() == [1, 3, 0] and e[3].tolist() == [0, 1, 2]
        if scores == "sigmoid":
            assert e[1].tolist() == [5, 0, 1] and w[1, 0].isnan() and not w[1, 1:].isnan().any()
            assert e[2].tolist() == [5, 0, 1] and w[2, 0] == 1
            assert e[5].tolist() == [2, 6, 0]
        else:
            assert w[1].isnan().all() and w[2].isnan().all() and w[5].isnan().all()
            assert w[3].tolist() == [1.0, 0.0, 0.0]
    # a number twice in the caller's own choice: both gradients
    op = binding.CRoute(0, 1, 1, 4, 3, 1, 1, 0, 1.0)
    e, g, z, dz = torch.tensor([[2, 2, 7]]), torch.tensor([[1.0, 2.0, 4.0]]), torch.zeros(1, 4), torch.empty(1, 4)
    assert lib.tt_route_backward(ctypes.byref(op), z.data_ptr(), e.data_ptr(), g.data_ptr(), dz.data_ptr(), None) == 0
    assert dz.tolist() == [[0.0, 0.0, 0.75, 0.0]]


# rows of logits whose scores leave the range of fp32, and what is added to choose them: (logits, bias, scores)
FAR_ROUTES = [([-88.0, -87.5, -89.0, -90.0], None, "sigmoid"), ([-89.0, -90.0, -200.0, -201.0], None, "sigmoid"), ([-100.0, -100.5, -700.0, -99.0], None, "sigmoid"),
              ([90.0, 101.0, 300.0, 89.0], None, "sigmoid"), ([0.0, -90.0, -90.5, -200.0], [-math.inf, 0, 0, 0], "softmax"),
              ([0.0, -120.0, -121.0, -500.0], [-2.0, 0, 0, 0], "softmax"), ([0.0, -95.0, -95.25, -94.0], [-2.0, 0, 0, -2.0], "softmax"),
              ([0.0, -600.0, -601.0, -650.0], [-2.0, 0, 0, 0], "softmax"), ([3.0, 2.5, -400.0, 1.0], None, "softmax"), ([500.0, 499.0, 0.0, -500.0], None, "softmax")]


@pytest.mark.parametrize("logits,bias,scores", FAR_ROUTES)
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("num,dtype", [(4, F32), (26, F32), (64, BF16), (100, F32), (700, F32)])
def test_route_of_scores_outside_single_precision(lib, logits, bias, scores, renorm, num, dtype):
    """Weights and their gradient where the chosen scores are too small for fp32: what 64 bits give.  The rest of the experts is masked."""
    from paper_2507_14668_amd import binding
    at = torch.arange(4) * (num // 4)
    z, b = torch.full((3, num), -math.inf), torch.zeros(num)
    z[:, at] = torch.tensor(logits)
    z = z.to(dtype)
    b[at] = torch.tensor(bias or [0.0] * 4)
    g = torch.tensor([[3.0, -2.0], [1e30, 1.0], [0.25, 0.25]])
    op = binding.CRoute(DT[dtype], binding.SCORES[scores], 3, num, 2, 1, 1, int(renorm), 2.5)
    how = dict(scores=scores, renormalize=renorm, scale=2.5)
    e, w, dz = Guarded((3, 2), torch.int64), Guarded((3, 2), F32), Guarded((3, num), dtype)
    gz, gb, gg = place(z), place(b[None]), place(g)
    assert lib.tt_route_forward(ctypes.byref(op), gz.ptr, gb.ptr, e.ptr, w.ptr, None) == 0
    want_w, want_e = ref.route64(z, 2, b, **how)
    assert torch.equal(e.t, want_e)
    ref.check(w.t, want_w, ref.weights_tol(want_w), "weights")
    assert lib.tt_route_backward(ctypes.byref(op), gz.ptr, e.ptr, gg.ptr, dz.ptr, None) == 0
    ref.check(dz.t, *ref.route_backward_wide64(z, e.t, g, **how), "dlogits")
    intact(gz, gb, gg, e, w, dz)


def test_route_gradients_show_what_is_not_a_number(lib):
    """A NaN or +infinity among the logits: NaN in a softmax row's gradient, as in its weights; scores that are zero in 64 bits have none."""
    from paper_2507_14668_amd import binding
    z = torch.zeros(4, 8)
    z[0, 5], z[1, 5], z[2, 1:] = math.nan, math.inf, -1e4
    e, g, dz = torch.tensor([[0, 1], [0, 5], [2, 3], [2, 3]]), torch.ones(4, 2), torch.empty(4, 8)
    g[:, 0] = 2.0
    for renorm in (0, 1):
        op = binding.CRoute(0, 0, 4, 8, 2, 1, 1, renorm, 1.0)
        assert lib.tt_route_backward(ctypes.byref(op), z.data_ptr(), e.data_ptr(), g.data_ptr(), dz.data_ptr(), None) == 0
        assert dz[0].isnan().all() and dz[1].isnan().all() and not dz[2].any()
        ref.check(dz[3:], *ref.route_backward_wide64(z[3:], e[3:], g[3:], "softmax", bool(renorm)), "dlogits")


def test_route_refusals(lib):
    from paper_2507_14668_amd import binding
    z, b, e, w, dz = torch.zeros(4, 8), torch.zeros(8), torch.zeros(4, 2, dtype=torch.int64), torch.zeros(4, 2), torch.zeros(4, 8)
    inval, shape = binding.TT_ERR_INVALID_ARG, binding.TT_ERR_SHAPE

    def call(z=z.data_ptr(), b=b.data_ptr(), e=e.data_ptr(), w=w.data_ptr(), **kw):
        op = binding.CRoute(0, 0, 4, 8, 2, 1, 1, 1, 1.0)
        for k, v in kw.items():
            setattr(op, k, v)
        return lib.tt_route_forward(ctypes.byref(op), z, b, e, w, None)
    assert call() == 0
    for bad in (dict(z=None), dict(e=None), dict(w=None), dict(z=z.data_ptr() + 1), dict(e=e.data_ptr() + 4), dict(b=b.data_ptr() + 2), dict(w=b.data_ptr()),
                dict(e=z.data_ptr()), dict(w=e.data_ptr()), dict(dtype=7), dict(scores=2), dict(rows=-1), dict(renormalize=2), dict(scale=math.inf), dict(scale=math.nan)):
        assert call(**bad) == inval, bad
    for bad in (dict(experts=0), dict(experts=1025), dict(choices=0), dict(choices=9), dict(groups=3), dict(groups=0), dict(top_groups=2), dict(top_groups=0),
                dict(groups=8, top_groups=1), dict(ld_logits=7), dict(rows=2 ** 30)):
        assert call(**bad) == shape, bad
    op = binding.CRoute(0, 0, 4, 8, 2, 1, 1, 1, 1.0)
    back = lambda z=z.data_ptr(), e=e.data_ptr(), g=w.data_ptr(), d=dz.data_ptr(): lib.tt_route_backward(ctypes.byref(op), z, e, g, d, None)
    assert back() == 0
    for bad in (dict(z=None), dict(e=None), dict(g=None), dict(d=None), dict(d=z.data_ptr()), dict(d=w.data_ptr())):
        assert back(**bad) == inval, bad


@pytest.mark.parametrize("rows,k,num", [(0, 3, 5), (1, 1, 1), (1, 2, 64), (40, 4, 7), (700, 3, 26), (300, 8, 1024), (8192, 1, 3), (2049, 4, 100), (4500, 3, 1000)])
@pytest.mark.parametrize("spread", [True, False])
def test_expert_order(lib, rows, k, num, spread):
    gen = torch.Generator().manual_seed(rows + num)
    e = torch.randint(-1, num + 1, (rows, k), generator=gen) if spread else torch.full((rows, k), num // 2, dtype=torch.int64)
    if spread and rows > 10:
        e[3], e[4] = 2 ** 40, -2 ** 63
    offsets, slots, sources = (Guarded((1, max(1, n)), t) for n, t in ((num + 1, torch.int64), (rows * k, torch.int32), (rows * k, torch.int32)))
    need = lib.tt_expert_order_workspace_bytes(rows * k, num)
    assert (need > 0) == (rows * k > 8192)
    ge, ws = place(e) if rows else Guarded((1, 1), torch.int64), Guarded((1, max(1, need)), torch.uint8)
    assert lib.tt_expert_order(ge.ptr, rows * k, num, offsets.ptr, slots.ptr, sources.ptr, ws.ptr, need, None) == 0
    want = ref.order_ref(e, num)
    assert torch.equal(offsets.t[0], want[0])
    if rows:
        assert torch.equal(slots.t[0].view(rows, k), want[1]) and torch.equal(sources.t[0], want[2])
    intact(offsets, slots, sources, ge, ws)


def test_expert_order_refusals(lib):
    from paper_2507_14668_amd import binding
    e, o = torch.zeros(20000, dtype=torch.int64), torch.zeros(9, dtype=torch.int64)
    s, t, ws = torch.zeros(20000, dtype=torch.int32), torch.zeros(20000, dtype=torch.int32), torch.zeros(1 << 16, dtype=torch.uint8)
    at = ws.data_ptr() + -ws.data_ptr() % 256

    def call(e=e.data_ptr(), n=20000, num=8, o=o.data_ptr(), s=s.data_ptr(), t=t.data_ptr(), ws=at, size=1 << 15):
        return lib.tt_expert_order(e, n, num, o, s, t, ws, size, None)
    assert call() == 0
    for bad in (dict(e=None), dict(o=None), dict(s=None), dict(t=None), dict(n=-1), dict(t=s.data_ptr()), dict(o=e.data_ptr()), dict(s=e.data_ptr()), dict(e=e.data_ptr() + 4)):
        assert call(**bad) == binding.TT_ERR_INVALID_ARG, bad
    for bad in (dict(num=0), dict(num=1025), dict(n=2 ** 31 - 1)):
        assert call(**bad) == binding.TT_ERR_SHAPE, bad
    for bad in (dict(ws=None), dict(ws=at + 8), dict(size=64)):
        assert call(**bad) == binding.TT_ERR_WORKSPACE, bad


# ---- the experts' rows
@pytest.mark.parametrize("rows,k,num,n,dtype,pad,shift", [
    (1, 1, 1, 1, F32, 0, 0), (5, 2, 3, 16, BF16, 0, 0), (37, 3, 5, 33, F16, 3, 1), (20, 4, 6, 130, F32, 0, 0), (9, 8, 16, 1000, BF16, 8, 0),
    (3, 2, 4, 2100, F32, 0, 0), (70, 1, 9, 64, F32, 0, 0)])
@pytest.mark.parametrize("weighted", [True, False])
def test_expert_rows_and_combine(lib, rows, k, num, n, dtype, pad, shift, weighted):
    from paper_2507_14668_amd import binding
    gen = torch.Generator().manual_seed(rows + n)
    e = torch.randint(-1, num, (rows, k), generator=gen)
    if rows == 1:
        e[0, 0] = 0
    _, slots, sources = ref.order_ref(e, num)
    x, y, res, grad = (randn(gen, r, n, dtype=dtype) for r in (rows, rows * k, rows, rows))
    w = torch.rand(rows, k, generator=gen) if weighted else None
    y[(sources < 0)] = math.nan  # behind the last place: read by nobody
    op = binding.CDeal(DT[dtype], n, rows, k, 1, n + pad, n + pad, n + pad, n + pad)
    gx, gy, gr, gg = (place(t, n + pad, shift) for t in (x, y, res, grad))
    gs, gt, gw = place(slots), place(sources[None]), place(w)
    out = Guarded((rows * k, n), dtype, n + pad, offset=shift)
    want, some = ref.rows_ref(x, slots), sources >= 0
    assert lib.tt_expert_rows(ctypes.byref(op), gx.ptr, gs.ptr, gt.ptr, out.ptr, None) == 0
    assert torch.equal(out.t[some], want[some]) and not out.t[~some].any()
    op.zero_rest = 0
    left = Guarded((rows * k, n), dtype, n + pad)
    assert lib.tt_expert_rows(ctypes.byref(op), gx.ptr, gs.ptr, None, left.ptr, None) == 0
    assert torch.equal(left.t[some], want[some]) and bool((left.t[~some].contiguous().view(torch.uint8) == 0xFF).all())
    c = Guarded((rows, n), dtype, n + pad, offset=shift)
    want = ref.combine64(y, slots, w, res, grad)
    assert lib.tt_expert_combine(ctypes.byref(op), gy.ptr, gs.ptr, ptr(gw), gr.ptr, c.ptr, None) == 0
    ref.check(c.t, *want["out"], "out")
    assert lib.tt_expert_combine(ctypes.byref(op), gy.ptr, gs.ptr, ptr(gw), gr.ptr, gr.ptr, None) == 0  # in place of the residual
    assert torch.equal(gr.t, c.t)
    dy, dw = Guarded((rows * k, n), dtype, n + pad, offset=shift), Guarded((rows, k), F32)
    assert lib.tt_expert_combine_backward(ctypes.byref(op), gy.ptr, gs.ptr, gt.ptr, ptr(gw), gg.ptr, dy.ptr, dw.ptr, None) == 0
    ref.check(dy.t[some], want["dy"][0][some], want["dy"][1][some], "dy")
    assert not dy.t[~some].any()
    ref.check(dw.t, *want["dweights"], "dweights")
    alone = Guarded((rows, k), F32)
    assert lib.tt_expert_combine_backward(ctypes.byref(op), gy.ptr, gs.ptr, None, ptr(gw), gg.ptr, None, alone.ptr, None) == 0
    assert torch.equal(alone.t, dw.t)
    alone = Guarded((rows * k, n), dtype, n + pad)
    assert lib.tt_expert_combine_backward(ctypes.byref(op), None, gs.ptr, gt.ptr, ptr(gw), gg.ptr, alone.ptr, None, None) == 0
    assert torch.equal(alone.t, dy.t)
    intact(gx, gy, gr, gg, gs, gt, gw, out, left, c, dy, dw)


def test_places_outside_count_as_none(lib):
    from paper_2507_14668_amd import binding
    x, slots = torch.randn(2, 8), torch.tensor([[0, 99], [-7, 2]], dtype=torch.int32)
    sources = torch.tensor([0, -1, 3, 99], dtype=torch.int32)
    op = binding.CDeal(0, 8, 2, 2, 1)
    out, c = Guarded((4, 8), F32), Guarded((2, 8), F32)
    assert lib.tt_expert_rows(ctypes.byref(op), x.data_ptr(), slots.data_ptr(), sources.data_ptr(), out.ptr, None) == 0
    assert torch.equal(out.t, torch.stack([x[0], 0 * x[0], x[1], 0 * x[0]]))
    assert lib.tt_expert_combine(ctypes.byref(op), out.ptr, slots.data_ptr(), None, None, c.ptr, None) == 0
    assert torch.equal(c.t, x)
    intact(out, c)


def test_expert_rows_refusals(lib):
    from paper_2507_14668_amd import binding
    x, y, s, t, w = torch.zeros(4, 8), torch.zeros(8, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(8, dtype=torch.int32), torch.zeros(4, 2)
    out, dw = torch.zeros(8, 8), torch.zeros(4, 2)
    p = lambda v: v if v is None or isinstance(v, int) else v.data_ptr()

    def op(kw):
        o = binding.CDeal(0, 8, 4, 2, 1)
        for k in list(kw):
            if hasattr(o, k):
                setattr(o, k, kw.pop(k))
        return ctypes.byref(o)

    def rows(**kw):
        o = op(kw)
        a = dict(x=x, s=s, t=t, out=out, **{})
        a.update(kw)
        return lib.tt_expert_rows(o, p(a["x"]), p(a["s"]), p(a["t"]), p(a["out"]), None)

    def combine(**kw):
        o = op(kw)
        a = dict(y=y, s=s, w=w, r=None, out=out)
        a.update(kw)
        return lib.tt_expert_combine(o, p(a["y"]), p(a["s"]), p(a["w"]), p(a["r"]), p(a["out"]), None)

    def back(**kw):
        o = op(kw)
        a = dict(y=y, s=s, t=t, w=w, g=x, dy=out, dw=dw)
        a.update(kw)
        return lib.tt_expert_combine_backward(o, p(a["y"]), p(a["s"]), p(a["t"]), p(a["w"]), p(a["g"]), p(a["dy"]), p(a["dw"]), None)
    assert rows() == combine() == back() == 0
    inval, shape = binding.TT_ERR_INVALID_ARG, binding.TT_ERR_SHAPE
    for call in (rows, combine, back):
        for bad in (dict(dim=0), dict(dim=(1 << 20) + 1), dict(choices=0), dict(choices=65), dict(ld_rows=7), dict(ld_places=7), dict(ld_dy=3), dict(rows=2 ** 30)):
            assert call(**bad) == shape, (call, bad)
        for bad in (dict(dtype=3), dict(rows=-1), dict(s=None), dict(s=s.data_ptr() + 2)):
            assert call(**bad) == inval, (call, bad)
    for bad in (dict(x=None), dict(out=None), dict(t=None), dict(out=x), dict(out=s), dict(x=x.data_ptr() + 1)):
        assert rows(**bad) == inval, bad
    for bad in (dict(y=None), dict(out=None), dict(out=y), dict(out=w), dict(r=out, ld_residual=16), dict(w=w.data_ptr() + 1)):
        assert combine(**bad) == inval, bad
    for bad in (dict(y=None), dict(g=None), dict(t=None), dict(dy=y), dict(dy=x), dict(dw=w), dict(dw=out)):
        assert back(**bad) == inval, bad


# ---- the loss
LOSSES = [
    # rows, dim, classes, dtype, bias, reduction, ignored, pad, shift
    (1, 1, 1, F32, False, "mean", 0, 0, 0),
    (1, 16, 70, BF16, True, "sum", 0, 0, 0),
    (5, 24, 300, F32, True, "mean", 2, 0, 0),
    (33, 33, 129, F16, True, "none", 5, 3, 1),
    (70, 16, 65, BF16, False, "mean", 10, 8, 0),
    (130, 64, 600, BF16, True, "mean", 20, 0, 0),
    (130, 40, 521, F16, False, "none", 0, 0, 0),
    (270, 128, 300, BF16, True, "mean", 30, 0, 0),
    (40, 100, 700, BF16, True, "none", 4, 0, 1),
    (140, 133, 500, F16, True, "mean", 4, 0, 1),  # a copy of W in longer rows
    (150, 136, 450, F32, True, "sum", 4, 0, 0),
    (66, 20, 40, F32, False, "none", 60, 1, 0),
    (9, 8, 20, F32, True, "mean", 9, 0, 0),       # no row counts
    (9, 8, 2000, BF16, True, "mean", 9, 0, 0),
    (300, 72, 264, F16, True, "sum", 3, 0, 0),
    (0, 8, 20, F32, True, "mean", 0, 0, 0),
    (20, 200, 1100, F32, True, "mean", 3, 0, 1),  # fp32 logits through memory: few rows, more classes than a wavefront takes,
    (1, 133, 2049, F32, True, "sum", 0, 2, 0),
    (70, 600, 130, F32, True, "none", 9, 0, 0),   # ... and sums in pieces
    (90, 1030, 70, F32, False, "mean", 90, 0, 0),
]


@pytest.mark.parametrize("rows,dim,classes,dtype,biased,reduction,ignored,pad,shift", LOSSES)
def test_cross_entropy(loss_lib, rows, dim, classes, dtype, biased, reduction, ignored, pad, shift):
    from paper_2507_14668_amd import binding
    lib, gen = loss_lib, torch.Generator().manual_seed(rows + classes)
    x, w = randn(gen, rows, dim, dtype=dtype), randn(gen, classes, dim, std=2 * dim ** -0.5, dtype=dtype)
    b = randn(gen, classes, dtype=dtype) if biased else None
    if biased and classes > 8:
        b[3] = -math.inf  # a class that is left out
    labels = torch.randint(0, classes, (rows,), generator=gen)
    labels[labels == 3] = 0
    skip = torch.randperm(rows, generator=gen)[:ignored]
    labels[skip] = -7
    x[skip] = math.nan  # nobody looks at them
    grad = randn(gen, rows) if reduction == "none" else torch.tensor(1.0 if dtype != F16 else 300.0)
    op = binding.CLoss(DT[dtype], binding.REDUCTIONS[reduction], rows, dim, classes, -7, dim + pad, dim + pad)
    gx, gw, gb, gl = place(x, dim + pad, shift), place(w, None, shift), place(b[None] if biased else None, None, shift), place(labels[None])
    gg = place(grad.reshape(1, -1))
    loss, lse = Guarded((1, max(1, rows if reduction == "none" else 1)), F32), Guarded((max(1, rows), 2), F32)
    want = ref.loss64(torch.where(torch.isnan(x), torch.zeros_like(x), x), w, labels, b, -7, reduction, grad) if rows else None
    ws = Guarded((1, lib.tt_cross_entropy_workspace_bytes(ctypes.byref(op), 0)), torch.uint8)
    assert lib.tt_cross_entropy_forward(ctypes.byref(op), gx.ptr, gw.ptr, ptr(gb), gl.ptr, loss.ptr, lse.ptr, ws.ptr, ws.cols, None) == 0
    ws2 = Guarded((1, lib.tt_cross_entropy_workspace_bytes(ctypes.byref(op), 1)), torch.uint8)
    dx, dw, db = Guarded((rows, dim), dtype, dim + pad, offset=shift), Guarded((classes, dim), dtype, offset=shift), Guarded((1, classes), dtype, offset=shift)
    back = lambda dx, dw, db: lib.tt_cross_entropy_backward(ctypes.byref(op), gx.ptr, gw.ptr, ptr(gb), gl.ptr, lse.ptr, gg.ptr, dx, dw, db, ws2.ptr, ws2.cols, None)
    assert back(dx.ptr, dw.ptr, db.ptr) == 0
    if rows:
        ref.check(loss.t[0] if reduction == "none" else loss.t[0, 0], *want["loss"], "loss")
        ref.check(lse.t[:, 0], *want["lse"], "lse")
        ref.check(dx.t, *want["dx"], "dx")
        ref.check(dw.t, *want["dw"], "dw")
        ref.check(db.t[0], *want["dbias"], "dbias")
        assert not dx.t[skip].any()
        for which in range(3):  # each by itself gives the same
            alone = [Guarded(tuple(t.t.shape), dtype, t.ld) if i == which else None for i, t in enumerate((dx, dw, db))]
            assert back(*[ptr(t) for t in alone]) == 0
            got, was = alone[which].t, (dx, dw, db)[which].t
            assert torch.equal(got, was) or which == 2 and torch.allclose(got.float(), was.float(), rtol=2 * torch.finfo(dtype).eps, atol=1e-6)
    else:
        assert loss.t[0, 0] == 0 and not dw.t.any() and not db.t.any()
    intact(gx, gw, gb, gl, gg, loss, lse, ws, ws2, dx, dw, db)


def test_cross_entropy_bad_labels(lib):
    """A label outside gives NaN, in its row's loss and in the gradients; ignore_index inside the classes is ignored."""
    from paper_2507_14668_amd import binding
    gen = torch.Generator().manual_seed(0)
    x, w = randn(gen, 4, 8), randn(gen, 10, 8)
    op = binding.CLoss(0, 0, 4, 8, 10, 3)
    ws = Guarded((1, max(lib.tt_cross_entropy_workspace_bytes(ctypes.byref(op), i) for i in (0, 1))), torch.uint8)
    for bad in (10, -1, 2 ** 40, -2 ** 63):
        labels, loss, lse = torch.tensor([1, bad, 3, 9]), torch.empty(4), torch.empty(4, 2)
        call = (ctypes.byref(op), x.data_ptr(), w.data_ptr(), None, labels.data_ptr())
        assert lib.tt_cross_entropy_forward(*call, loss.data_ptr(), lse.data_ptr(), ws.ptr, ws.cols, None) == 0
        want = ref.loss64(x[[0, 3]], w, labels[[0, 3]], ignore_index=3, reduction="none")
        ref.check(loss[[0, 3]], *want["loss"], "loss")
        assert loss[1].isnan() and loss[2] == 0
        grad, dx, dw = torch.ones(4), torch.empty(4, 8), torch.empty(10, 8)
        assert lib.tt_cross_entropy_backward(*call, lse.data_ptr(), grad.data_ptr(), dx.data_ptr(), dw.data_ptr(), None, ws.ptr, ws.cols, None) == 0
        assert dx[1].isnan().all() and not dx[[0, 2, 3]].isnan().any() and dw.isnan().all() and not dx[2].any()


def test_cross_entropy_special_logits(lib):
    """Large logits, a masked label, no class at all, NaN and infinities in a row."""
    from paper_2507_14668_amd import binding
    w, b = torch.eye(4), torch.tensor([0.0, 0.0, 0.0, -math.inf])
    x = torch.tensor([[1e4, 0, 0, 0], [1e4, 0, 0, 0], [0, 0, 0, 5], [0, math.nan, 0, 0], [0, math.inf, 0, 0], [-3e38, 3e38, 0, 0]])
    labels = torch.tensor([0, 1, 3, 0, 0, 1])
    op = binding.CLoss(0, 0, 6, 4, 4, -100)
    ws = Guarded((1, lib.tt_cross_entropy_workspace_bytes(ctypes.byref(op), 0)), torch.uint8)
    loss, lse = torch.empty(6), torch.empty(6, 2)
    assert lib.tt_cross_entropy_forward(ctypes.byref(op), x.data_ptr(), w.data_ptr(), b.data_ptr(), labels.data_ptr(), loss.data_ptr(), lse.data_ptr(), ws.ptr,
                                        ws.cols, None) == 0
    # a logit to units of log 2 and back is two constants and two products, each off by half a step of 2^-23, and the logarithm of a sum near
    # one is off by the sum's half step: 4 x 2^-24 of the value and 2^-24
    near = lambda got, want: abs(float(got) - want) <= 2.0 ** -22 * abs(want) + 2.0 ** -24
    assert near(loss[0], 0) and near(loss[1], 1e4) and loss[2] == math.inf and loss[3].isnan() and loss[4].isnan() and near(loss[5], 0)
    b[:] = -math.inf
    assert lib.tt_cross_entropy_forward(ctypes.byref(op), x.data_ptr(), w.data_ptr(), b.data_ptr(), labels.data_ptr(), loss.data_ptr(), lse.data_ptr(), ws.ptr,
                                        ws.cols, None) == 0
    assert loss.isnan().all()


@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
@pytest.mark.parametrize("dim,dtype", [(64, F32), (64, BF16), (100, BF16), (128, F32), (136, BF16), (200, F32), (200, BF16)])
def test_cross_entropy_of_large_operands(lib, dim, dtype, reduction):
    """Rows, then classes, near the type's largest number, and logits of ordinary size: gradients that the type holds are not lost on the way.  A row's numbers are `size` in one
    column and 2 / size in another (a quarter for the second class), the classes' the other way round; each logit is one product of them, or two."""
    from paper_2507_14668_amd import binding
    size, up, classes = 2.0 ** 125, 2.0 ** -125, 9
    for first, second in ((size, up), (up, size)):
        x, w = torch.zeros(3, dim), torch.zeros(classes, dim)
        x[0, 1], x[1, 1], x[2, 20] = first, -first, first / 2
        w[2, 1], w[3, 1], w[4, 20] = 2 * second, -second, second / 2
        labels = torch.tensor([2, 3, 4])
        x, w = x.to(dtype), w.to(dtype)
        grad = torch.ones(3 if reduction == "none" else 1)
        want = ref.loss64(x, w, labels, reduction=reduction, grad=grad if reduction == "none" else grad[0])
        op = binding.CLoss(DT[dtype], binding.REDUCTIONS[reduction], 3, dim, classes, -100)
        ws = Guarded((1, max(lib.tt_cross_entropy_workspace_bytes(ctypes.byref(op), i) for i in (0, 1))), torch.uint8)
        loss, stats, dx, dw, db = torch.empty(3), torch.empty(3, 2), torch.empty_like(x), torch.empty_like(w), torch.empty(classes, dtype=dtype)
        call = (ctypes.byref(op), x.data_ptr(), w.data_ptr(), None, labels.data_ptr())
        assert lib.tt_cross_entropy_forward(*call, loss.data_ptr(), stats.data_ptr(), ws.ptr, ws.cols, None) == 0
        assert lib.tt_cross_entropy_backward(*call, stats.data_ptr(), grad.data_ptr(), dx.data_ptr(), dw.data_ptr(), db.data_ptr(), ws.ptr, ws.cols, None) == 0
        ref.check(loss if reduction == "none" else loss[0], *want["loss"], "loss")
        small = 2.0 ** -100 if dtype == F32 else 0.0  # (short fp32 rows: numbers below 2^-100 may have fewer bits)
        for got, name in ((dx, "dx"), (dw, "dw"), (db, "dbias")):
            ref.check(got, want[name][0], want[name][1] + small, name)


LARGE = [2.0 ** 12, 2.0 ** 20, 2.0 ** 24, 2.0 ** 27, 2.0 ** 32, 1e19, 2.0 ** 100, 1e38]


def large_logits(size, dim, dtype, biased):
    """x, w, bias and labels of rows whose largest logits are `size` and 1.5 times that (rounded to the type), nothing near them: every probability is 0 or 1."""
    classes, scale = 40, 2.0 ** 10  # (a logit is one product)
    z = torch.zeros(7, classes)
    z[0, 5], z[0, 9] = size, 1.5 * size
    z[1, 5], z[1, 9] = size, 1.5 * size
    z[2], z[2, 30] = -1.5 * size, -size
    z[3], z[3, 30] = -1.5 * size, -size
    z[4, 17] = size
    z[5, 17] = -size
    z[5, 18] = size
    z[6, 39], z[6, 0] = 1.25 * size, -size
    labels = torch.tensor([5, 9, 0, 30, 3, 17, 39])
    x, w, b = torch.zeros(7, dim), torch.zeros(classes, dim), None
    w[torch.arange(classes), torch.arange(classes)] = scale
    x[:, :classes] = z / scale
    if biased:  # the same logits, less what the bias has
        b = torch.zeros(classes)
        b[9], b[30] = size / 4, size / 4
    return x.to(dtype), w.to(dtype), None if b is None else b.to(dtype), labels


def large_logits64(x, w, b, labels, grad):
    """loss, dx, dw and dbias in 64 bits with their tolerances: one product and one sum make a logit, and G is exact, so that fp32 rounds a logit twice, the loss twice more, and
    sums over rows by 2 (rows + 2) u of their terms."""
    dtype, x, w = x.dtype, x.double(), w.double()
    bias = torch.zeros(w.shape[0], dtype=torch.float64) if b is None else b.double()
    z = x @ w.t() + bias
    lse, zl = torch.logsumexp(z, 1), z.gather(1, labels[:, None])[:, 0]
    G = (torch.exp(z - lse[:, None]) - torch.zeros_like(z).scatter_(1, labels[:, None], 1.0)) * grad.double()[:, None]
    assert bool(((G == 0) | (G.abs() == grad.double().abs()[:, None])).all())
    result = dict(loss=(lse - zl, 2 * ref.U * (2 * (lse - zl).abs() + lse.abs() * (b is not None) + zl.abs() * (b is not None))))
    for name, a, c in (("dx", G, w), ("dw", G.t(), x), ("dbias", G.t(), torch.ones(x.shape[0], 1, dtype=torch.float64))):
        v, size = a @ c, a.abs() @ c.abs()
        result[name] = (v, 2 * (x.shape[0] + 2) * ref.U * size + ref.rounding(v, dtype))
    return result


@pytest.mark.parametrize("size", LARGE)
@pytest.mark.parametrize("dim,dtype", [(64, F32), (64, BF16), (50, F16), (100, BF16), (128, F32), (136, BF16), (200, F32)])
@pytest.mark.parametrize("biased,reduction", [(False, "none"), (True, "none"), (True, "sum")])
def test_cross_entropy_of_large_logits(lib, size, dim, dtype, biased, reduction):
    """Finite logits of any size, far apart: losses to fp32's precision and never below zero, gradients of zeros and ones."""
    from paper_2507_14668_amd import binding
    if dtype == F16:
        size = min(size, 2.0 ** 24 if not biased else 2.0 ** 14)
    x, w, b, labels = large_logits(size, dim, dtype, biased)
    grad = torch.tensor([1.0, -2.0, 0.5, 1.0, 3.0, 1.0, 0.25]) if reduction == "none" else torch.ones(7)
    want = large_logits64(x, w, b, labels, grad)
    gx, gw, gb, gl, gg = place(x), place(w), place(None if b is None else b[None]), place(labels[None]), place(grad[None, :7 if reduction == "none" else 1])
    op = binding.CLoss(DT[dtype], binding.REDUCTIONS[reduction], 7, dim, 40, -100)
    ws = Guarded((1, max(lib.tt_cross_entropy_workspace_bytes(ctypes.byref(op), i) for i in (0, 1))), torch.uint8)
    loss, stats = Guarded((1, 7), F32), Guarded((7, 2), F32)
    dx, dw, db = Guarded((7, dim), dtype), Guarded((40, dim), dtype), Guarded((1, 40), dtype)
    call = (ctypes.byref(op), gx.ptr, gw.ptr, ptr(gb), gl.ptr)
    assert lib.tt_cross_entropy_forward(*call, loss.ptr, stats.ptr, ws.ptr, ws.cols, None) == 0
    assert lib.tt_cross_entropy_backward(*call, stats.ptr, gg.ptr, dx.ptr, dw.ptr, db.ptr, ws.ptr, ws.cols, None) == 0
    assert bool((stats.t[:, 1] >= 0).all())
    ref.check(stats.t[:, 1], *want["loss"], "loss")
    beyond = 2.0 ** 16 if dtype == F16 else math.inf  # (what rounds to fp16's infinity: 3 times 2^24 / 2^10 and more)
    for got, name in ((dx.t, "dx"), (dw.t, "dw"), (db.t.t(), "dbias")):
        ref.check(got.float().clamp(-beyond, beyond), *want[name], name)
    intact(gx, gw, gb, gl, gg, ws, stats, dx, dw, db)


@pytest.mark.parametrize("std", [20.0, 60.0])
@pytest.mark.parametrize("dim", [64, 128])
def test_cross_entropy_gradients_of_rows_and_classes_are_as_good(lib, dim, std):
    """fp32, short rows, an lse of some ten to hundred: dx, dW and dbias come of the same softmax.  A probability is off by the error of a logit (twice dim + 2 units of the sum of its terms'
    sizes, 6 for the parts' dropped terms), of lse (its own rounding, and a row's error of the same kind) and of exp2's argument; G's errors go into the sums in the 2-norm
    no more than G's size times that; the sums add rows + 2 and classes + 2 units.  Chains that started at -lse lost ulp(lse) at every step: 2e-5 and 6e-5."""
    from paper_2507_14668_amd import binding
    gen = torch.Generator().manual_seed(dim)
    rows, classes = 48, 700
    x, w, labels = randn(gen, rows, dim), randn(gen, classes, dim, std=std * dim ** -0.5), torch.randint(0, classes, (rows,), generator=gen)
    z = x.double() @ w.double().t()
    lse, grad = torch.logsumexp(z, 1), torch.ones(1)
    G = torch.softmax(z, 1)
    G[torch.arange(rows), labels] = -(1 - G[torch.arange(rows), labels])
    op = binding.CLoss(0, binding.REDUCTIONS["sum"], rows, dim, classes, -100)
    ws = Guarded((1, max(lib.tt_cross_entropy_workspace_bytes(ctypes.byref(op), i) for i in (0, 1))), torch.uint8)
    loss, stats, dx, dw, db = torch.empty(1), torch.empty(rows, 2), torch.empty_like(x), torch.empty_like(w), torch.empty(classes)
    call = (ctypes.byref(op), x.data_ptr(), w.data_ptr(), None, labels.data_ptr())
    assert lib.tt_cross_entropy_forward(*call, loss.data_ptr(), stats.data_ptr(), ws.ptr, ws.cols, None) == 0
    assert lib.tt_cross_entropy_backward(*call, stats.data_ptr(), grad.data_ptr(), dx.data_ptr(), dw.data_ptr(), db.data_ptr(), ws.ptr, ws.cols, None) == 0
    # random roundings of a chain of dim / 8 additions of partial sums up to |z| (the instruction adds eight products at a time): sqrt of their number, three deviations
    logit = 3 * ref.U * math.sqrt(dim / 8 * 6) * float(z.abs().max())
    most = 2 * logit + 2 * ref.U * float(lse.max()) + 32 * ref.U
    off = {}
    for got, want, name in ((dx, G @ w.double(), "dx"), (dw, G.t() @ x.double(), "dw"), (db, G.sum(0), "dbias")):
        off[name] = float((got.double() - want).norm() / want.norm())
        assert off[name] <= most, (name, off, most)
    assert max(off.values()) <= 8 * off["dx"] + 8 * ref.U, off


# a row's label's logit and the others' (all classes, then the first ones): sure of its label by 3 to 60, near zero and near 1000
SURE = [(3.0, 0.0, []), (8.0, 0.0, [-1.0, 0.5]), (10.5, 0.0, [1.0]), (11.0, 0.0, []), (11.5, 0.0, [0.25, -3.0]), (17.0, -2.0, [1.0]), (24.0, 0.0, []), (40.0, -1.0, [2.0]), (60.0, 0.0, []),
        (1000.0, 992.0, []), (1000.0, 960.0, [988.0]), (-8.0, -20.0, [-16.0]), (0.0, 0.0, []), (-5.0, 1.0, [7.0, 7.0])]


def sure_rows(dim, dtype, label):
    """x, w and labels with exactly the logits above: a logit is one product with 1."""
    classes = 64
    x, w = torch.zeros(len(SURE), dim), torch.zeros(classes, dim)
    w[torch.arange(classes), torch.arange(classes)] = 1.0
    for r, (own, rest, more) in enumerate(SURE):
        x[r, :classes] = rest
        x[r, :len(more)] = torch.tensor(more)
        x[r, label] = own
    return x.to(dtype), w.to(dtype), torch.full((len(SURE),), label)


def sure_rows64(x, w, labels):
    """Losses and G in 64 bits, and their errors relative to their size: the exponent of what the others have beside the label is off by u of itself for the difference, as much for its scaling and as
    much for m, the sum has 64 terms and three joins, exp, log1p and expm1 add a few units (in all 2 |difference| + 80 u); an lse is rounded by u of itself, and so are differences to it."""
    z = x.double() @ w.double().t()
    at = torch.arange(x.shape[0])
    own = z[at, labels]
    d = z - own[:, None]
    d[at, labels] = -math.inf
    loss = torch.log1p(torch.exp(d).sum(1))
    G = torch.exp(z - (own + loss)[:, None])
    G[at, labels] = torch.expm1(-loss)
    far = d.amax(1).abs()
    rel = ref.U * (2 * far + 80)
    each = ref.U * (2 * (own + loss).abs()[:, None] + 2 * (z - (own + loss)[:, None]).abs() + 16)
    each[at, labels] = rel
    return loss, rel * loss, G, each * G.abs()


@pytest.mark.parametrize("dim,dtype", [(64, F32), (64, BF16), (80, F16), (128, F32), (128, BF16), (136, F32), (136, BF16), (200, F16)])
@pytest.mark.parametrize("label", [50, 3])
def test_cross_entropy_of_sure_rows(loss_lib, dim, dtype, label):
    """Row by row: losses and gradients of rows that are nearly sure of their label keep their relative precision, however small they are, in a late step of the classes too."""
    from paper_2507_14668_amd import binding
    x, w, labels = sure_rows(dim, dtype, label)
    rows, classes = x.shape[0], w.shape[0]
    loss64, eloss, G, eG = sure_rows64(x, w, labels)
    eps = torch.finfo(dtype).eps / 2
    if dtype != F32:  # G to 16 bits (fp16: smallest steps of 2^-37), and the result
        eG = eG + 2.01 * eps * G.abs() + (2.0 ** -37 if dtype == F16 else 2.0 ** -133)
    loss, stats, dx, dw, db = torch.empty(rows), torch.empty(rows, 2), torch.empty_like(x), torch.empty_like(w), torch.empty(classes, dtype=dtype)
    grad = torch.ones(rows)
    for r in [None, 4, 8]:  # all of them; one row alone, whose gradient dbias then is
        if r is not None:
            labels = torch.full_like(labels, -100)
            labels[r] = label
        op = binding.CLoss(DT[dtype], 0, rows, dim, classes, -100)
        ws = Guarded((1, max(loss_lib.tt_cross_entropy_workspace_bytes(ctypes.byref(op), i) for i in (0, 1))), torch.uint8)
        call = (ctypes.byref(op), x.data_ptr(), w.data_ptr(), None, labels.data_ptr())
        assert loss_lib.tt_cross_entropy_forward(*call, loss.data_ptr(), stats.data_ptr(), ws.ptr, ws.cols, None) == 0
        assert loss_lib.tt_cross_entropy_backward(*call, stats.data_ptr(), grad.data_ptr(), dx.data_ptr(), dw.data_ptr(), db.data_ptr(), ws.ptr, ws.cols, None) == 0
        if r is None:
            ref.check(loss, loss64, eloss, "loss")
            want = torch.cat([G, torch.zeros(rows, dim - classes)], 1)  # (W is the unit matrix)
            ref.check(dx, want, torch.cat([eG, torch.zeros(rows, dim - classes)], 1) + ref.rounding(want, dtype), "dx")
        else:
            ref.check(db, G[r], eG[r] + ref.rounding(G[r], dtype), "dbias")


@pytest.mark.parametrize("dim", [64, 128, 136, 200])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
@pytest.mark.parametrize("share", [math.inf, -math.inf, math.nan])
def test_cross_entropy_of_rows_that_do_not_count_under_any_gradient(lib, dim, dtype, reduction, share):
    """A loss scaler's overflow: rows that do not count have gradients of zero all the same, and so have the classes if no row counts."""
    from paper_2507_14668_amd import binding
    gen = torch.Generator().manual_seed(dim)
    x, w = randn(gen, 9, dim, dtype=dtype), randn(gen, 70, dim, std=dim ** -0.5, dtype=dtype)
    for some in (True, False):
        labels = torch.randint(0, 70, (9,), generator=gen)
        labels[[1, 4, 8]] = -100
        if not some:
            labels[:] = -100
        op = binding.CLoss(DT[dtype], binding.REDUCTIONS[reduction], 9, dim, 70, -100)
        ws = Guarded((1, max(lib.tt_cross_entropy_workspace_bytes(ctypes.byref(op), i) for i in (0, 1))), torch.uint8)
        loss, stats, dx, dw, db = torch.empty(9), torch.empty(9, 2), torch.empty_like(x), torch.empty_like(w), torch.empty(70, dtype=dtype)
        grad = torch.full((9,), share)
        call = (ctypes.byref(op), x.data_ptr(), w.data_ptr(), None, labels.data_ptr())
        assert lib.tt_cross_entropy_forward(*call, loss.data_ptr(), stats.data_ptr(), ws.ptr, ws.cols, None) == 0
        assert lib.tt_cross_entropy_backward(*call, stats.data_ptr(), grad.data_ptr(), dx.data_ptr(), dw.data_ptr(), db.data_ptr(), ws.ptr, ws.cols, None) == 0
        assert not dx[labels == -100].any() and (not some or not dx[labels != -100].isfinite().any())
        assert some or not dw.any() and not db.any()


def test_cross_entropy_refusals(lib):
    from paper_2507_14668_amd import binding
    x, w, b, lab, loss, lse = torch.zeros(4, 8), torch.zeros(10, 8), torch.zeros(10), torch.zeros(4, dtype=torch.int64), torch.zeros(4), torch.zeros(4, 2)
    ws = Guarded((1, 1 << 20), torch.uint8)
    p = lambda v: v if v is None or isinstance(v, int) else v.data_ptr()
    inval, shape, work = binding.TT_ERR_INVALID_ARG, binding.TT_ERR_SHAPE, binding.TT_ERR_WORKSPACE

    def make(kw):
        o = binding.CLoss(0, 0, 4, 8, 10, -100)
        for k in list(kw):
            if hasattr(o, k):
                setattr(o, k, kw.pop(k))
        return ctypes.byref(o)

    def forward(**kw):
        o = make(kw)
        a = dict(x=x, w=w, b=b, lab=lab, loss=loss, lse=lse, ws=ws.ptr, size=ws.cols)
        a.update(kw)
        return lib.tt_cross_entropy_forward(o, *(p(a[k]) for k in ("x", "w", "b", "lab", "loss", "lse", "ws")), a["size"], None)
    dx, dw, db, grad = torch.zeros(4, 8), torch.zeros(10, 8), torch.zeros(10), torch.zeros(4)

    def backward(**kw):
        o = make(kw)
        a = dict(x=x, w=w, b=b, lab=lab, lse=lse, grad=grad, dx=dx, dw=dw, db=db, ws=ws.ptr, size=ws.cols)
        a.update(kw)
        return lib.tt_cross_entropy_backward(o, *(p(a[k]) for k in ("x", "w", "b", "lab", "lse", "grad", "dx", "dw", "db", "ws")), a["size"], None)
    assert forward() == backward() == 0
    for call in (forward, backward):
        for bad in (dict(dim=0), dict(dim=(1 << 20) + 1), dict(classes=0), dict(classes=2 ** 30 + 1), dict(rows=2 ** 31 - 1), dict(ld_x=7), dict(ld_dx=7)):
            assert call(**bad) == shape, (call, bad)
        for bad in (dict(dtype=3), dict(reduce=3), dict(rows=-1), dict(x=None), dict(w=None), dict(lab=None), dict(lse=None), dict(x=x.data_ptr() + 1),
                    dict(lab=lab.data_ptr() + 4), dict(b=b.data_ptr() + 1)):
            assert call(**bad) == inval, (call, bad)
        for bad in (dict(ws=None), dict(ws=ws.ptr + 16), dict(size=100)):
            assert call(**bad) == work, (call, bad)
    for bad in (dict(loss=None), dict(loss=lse), dict(loss=x), dict(lse=w), dict(loss=lab)):
        assert forward(**bad) == inval, bad
    for bad in (dict(grad=None), dict(dx=x), dict(dw=w), dict(db=b), dict(dx=lse), dict(dw=dx), dict(db=dw), dict(dx=grad)):
        assert backward(**bad) == inval, bad
    assert lib.tt_cross_entropy_workspace_bytes(None, 0) == 0
