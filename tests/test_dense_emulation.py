"""The dense operators' host code and kernels compiled for the CPU (tests/cpu_emulation): values against 64 bits through the C
ABI, and every refusal of an argument.  Buffers sit between guards of ones that nothing may touch."""
import ctypes
import math
import os
import sys

import pytest
import torch

import dense_ref as ref

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "cpu_emulation"))
import build as emu_build  # noqa: E402

BUILD_DIR = os.path.join(os.path.dirname(os.path.abspath(__file__)), "cpu_emulation", "_build")
pytestmark = pytest.mark.skipif(not emu_build.available(), reason="host clang++ of the ROCm toolchain not found")
DT = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
GUARD = 512


NO_ROWS = {"tt_gemm_rows": ["-DTT_GEMM_FEW_ROWS=0"]}
VARIANTS = {"as it is": ("as_it_is", {}), "small tiles": ("small", NO_ROWS), "large tiles": ("large", dict(NO_ROWS, tt_gemm=["-DTT_GEMM_LARGE_TILES=1"])),
            "direct tiles": ("direct", dict(NO_ROWS, tt_gemm_direct=["-DTT_GEMM_DIRECT_TILES=1", "-DTT_GEMM_DIRECT_LEAST=0"]))}


@pytest.fixture(scope="module", params=VARIANTS)
def lib(request):
    """The library as it is (few rows mostly), without the kernel for few rows, and with the larger tiles from the first one on."""
    lib = ctypes.CDLL(emu_build.build_dense(BUILD_DIR, *VARIANTS[request.param]))
    vp, sz, f32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float
    lib.tt_dense_workspace_bytes.restype = lib.tt_orthogonalize_workspace_bytes.restype = lib.tt_core_ortho_workspace_bytes.restype = sz
    lib.tt_dense_workspace_bytes.argtypes = [vp, ctypes.c_int]
    lib.tt_dense_forward.argtypes = [vp] * 8 + [sz, vp]
    lib.tt_dense_backward.argtypes = [vp] * 9 + [sz, vp]
    lib.tt_orthogonalize_workspace_bytes.argtypes = lib.tt_core_ortho_workspace_bytes.argtypes = [vp]
    lib.tt_orthogonalize.argtypes = [vp, vp, vp, ctypes.c_int, vp, f32, vp, sz, vp]
    lib.tt_core_ortho_update.argtypes = [vp, vp, vp, f32, f32, ctypes.c_int, ctypes.c_int, vp, f32, vp, sz, vp]
    return lib


class Guarded:
    """Memory of `shape` with rows `ld` apart, every byte around it 0xFF before and after."""

    def __init__(self, shape, dtype, ld=None, align=256, offset=0):
        cols = shape[-1]
        ld = ld or cols
        rows = 1
        for s in shape[:-1]:
            rows *= s
        size = torch.empty(0, dtype=dtype).element_size()
        self.raw = torch.full((GUARD + align + offset * size + rows * ld * size + GUARD,), 0xFF, dtype=torch.uint8)
        at = GUARD + (-(self.raw.data_ptr() + GUARD)) % align + offset * size
        flat = self.raw[at:at + rows * ld * size].view(dtype)
        self.t = flat.view(rows, ld)[:, :cols] if len(shape) == 2 else flat.view(shape)
        self.ptr, self.at, self.ld, self.size, self.cols, self.rows = self.t.data_ptr(), at, ld, size, cols, rows

    def intact(self):
        raw = self.raw.clone()
        body = raw[self.at:self.at + self.rows * self.ld * self.size].view(self.rows, self.ld * self.size)
        body[:, :self.cols * self.size] = 0xFF
        return bool((raw == 0xFF).all())


def place(t, ld=None, offset=0):
    if t is None:
        return None
    g = Guarded(tuple(t.shape), t.dtype, ld, offset=offset)
    g.t.copy_(t)
    return g


def ptr(g):
    return None if g is None else g.ptr


def dense_op(x, w, act, offsets, zero_rest=0, **ld):
    from paper_2507_14668_amd import binding
    op = binding.CDense()
    op.dtype, op.activation, op.zero_rest = DT[x.dtype], binding.ACTIVATIONS[act], zero_rest
    op.rows, op.in_dim, op.out_dim = x.shape[0], w.shape[-1], w.shape[-2]
    if offsets is not None:
        op.groups, op.offsets = w.shape[0], offsets.data_ptr()
    for k, v in ld.items():
        setattr(op, k, v)
    return op


def make(rows, k, n, dtype, groups=0, seed=0):
    gen = torch.Generator().manual_seed(seed)
    lead = (groups,) if groups else ()
    f = lambda *s, std=1.0: (torch.randn(*s, generator=gen) * std).to(dtype)
    return f(rows, k), f(*lead, n, k, std=k ** -0.5), f(*lead, n), f(rows, n), f(rows, n)


CASES = [
    # rows, k, n, dtype, act, groups' offsets, pad, element offset
    (1, 1, 1, torch.float32, "none", None, 0, 0),
    (1, 8, 5, torch.bfloat16, "relu", None, 0, 0),
    (65, 33, 67, torch.float32, "gelu", None, 3, 1),
    (70, 40, 66, torch.bfloat16, "gelu", None, 0, 1),
    (64, 64, 64, torch.float16, "silu", None, 8, 0),
    (3, 131, 130, torch.float16, "sigmoid", None, 1, 3),
    (40, 17, 9, torch.float32, "silu", [0, 0, 13, 13, 40], 0, 0),
    (150, 24, 70, torch.bfloat16, "relu", [0, 70, 70, 150], 0, 0),
    (90, 9, 33, torch.float16, "gelu", [5, 8, 80], 2, 1),
    (30, 16, 16, torch.float32, "none", [0, 20, 10, 25], 0, 0),      # not in order: the running maximum counts
    (30, 16, 16, torch.bfloat16, "none", [-4, 12, 99], 0, 0),        # outside: clamped
    (600, 9, 12, torch.float32, "silu", [0, 20, 570, 600], 0, 0),    # a group whose sum over rows is cut
    (300, 72, 264, torch.bfloat16, "silu", [0, 130, 130, 299], 8, 0),
    (270, 136, 40, torch.float16, "relu", None, 0, 0),
    (20, 8, 8, torch.float32, "relu", [20, 20], 0, 0),               # one group, without rows
    (70, 8, 8, torch.float32, "none", [min(i, 70) for i in range(132)], 0, 0),  # 131 groups: more than a wavefront's lanes
]


@pytest.mark.parametrize("rows,k,n,dtype,act,offs,pad,shift", CASES)
@pytest.mark.parametrize("extras", [True, False])
def test_dense_values(lib, rows, k, n, dtype, act, offs, pad, shift, extras):
    groups = 0 if offs is None else len(offs) - 1
    offsets = None if offs is None else torch.tensor(offs, dtype=torch.int64)
    x, w, bias, res, grad = make(rows, k, n, dtype, groups)
    if not extras:
        bias = res = None
    gx, gw, gb, gr = place(x, k + pad, shift), place(w, None, shift), place(bias, None, shift), place(res, n + pad, shift)
    out, pre = Guarded((rows, n), dtype, n + pad, offset=shift), Guarded((rows, n), dtype, offset=shift)
    op = dense_op(x, w, act, offsets, ld_x=k + pad, ld_out=n + pad, ld_residual=n + pad)
    assert lib.tt_dense_workspace_bytes(ctypes.byref(op), 0) % 256 == 0
    ws = Guarded((1, max(1, lib.tt_dense_workspace_bytes(ctypes.byref(op), 0))), torch.uint8)
    assert lib.tt_dense_forward(ctypes.byref(op), gx.ptr, gw.ptr, ptr(gb), ptr(gr), out.ptr, pre.ptr, ws.ptr, ws.cols, None) == 0
    want, tol, z, tz = ref.forward64(x, w, bias, res, act, offsets)
    member = ~torch.isnan(z[:, 0])
    ref.check(out.t[member], want[member], tol[member], "out")
    ref.check(pre.t[member], z[member], tz[member], "pre")
    untouched = torch.full((1,), 0xFF, dtype=torch.uint8).expand(8)[:out.size].clone().contiguous()
    for t in (out, pre):  # rows of no group as they were
        rest = t.t[~member].contiguous().view(torch.uint8) if dtype != torch.float32 else t.t[~member].contiguous().view(torch.uint8)
        assert bool((rest == 0xFF).all()) and untouched.numel() == out.size
    for g in (gx, gw, gb, gr, out, pre, ws):
        assert g is None or g.intact()
    # cleared instead, and over the residual's own memory
    if extras:
        op.zero_rest = 1
        assert lib.tt_dense_forward(ctypes.byref(op), gx.ptr, gw.ptr, gb.ptr, gr.ptr, gr.ptr, None, ws.ptr, ws.cols, None) == 0
        assert torch.equal(gr.t[member], out.t[member]) and bool((gr.t[~member] == 0).all()) and gr.intact()

    # backward
    gg = place(grad, n + pad, shift)
    pz = place(z.nan_to_num(0).to(dtype), None, shift)
    (dx, dw, db), (tx, tw, tb) = ref.backward64(x, w, grad, pz.t, act, offsets)
    op = dense_op(x, w, act, offsets, zero_rest=1, ld_x=k + pad, ld_grad=n + pad, ld_dx=k + 2 * pad)
    need = lib.tt_dense_workspace_bytes(ctypes.byref(op), 1)
    ws = Guarded((1, need), torch.uint8)
    for mask in (7, 1, 2, 4, 6):
        ox = Guarded((rows, k), dtype, k + 2 * pad, offset=shift) if mask & 1 else None
        ow = Guarded(tuple(w.shape), dtype, offset=shift) if mask & 2 else None
        ob = Guarded(tuple(w.shape[:-1]), dtype, offset=shift) if mask & 4 else None
        assert lib.tt_dense_backward(ctypes.byref(op), gx.ptr if mask & 2 else None, gw.ptr if mask & 1 else None, pz.ptr if act != "none" else None,
                                     gg.ptr, ptr(ox), ptr(ow), ptr(ob), ws.ptr, need, None) == 0
        if ox:
            ref.check(ox.t[member], dx[member], tx[member], "dx")
            assert bool((ox.t[~member] == 0).all())
        if ow:
            ref.check(ow.t, dw, tw, "dw")
        if ob:
            ref.check(ob.t.view(db.shape), db, tb, "dbias")
        for g in (ox, ow, ob, gx, gw, gg, pz, ws):
            assert g is None or g.intact()


def test_dense_without_rows(lib):
    x, w, bias, _, _ = make(0, 8, 4, torch.float32)
    op = dense_op(x, w, "relu", None)
    assert lib.tt_dense_forward(ctypes.byref(op), None, None, None, None, None, None, None, 0, None) == 0
    need = lib.tt_dense_workspace_bytes(ctypes.byref(op), 1)
    ws, dw, db = Guarded((1, need), torch.uint8), Guarded((4, 8), torch.float32), Guarded((1, 4), torch.float32)
    assert lib.tt_dense_backward(ctypes.byref(op), None, None, None, None, None, dw.ptr, db.ptr, ws.ptr, need, None) == 0
    assert bool((dw.t == 0).all()) and bool((db.t == 0).all()) and dw.intact() and db.intact()
    # ... and of groups
    x, w, bias, _, _ = make(0, 8, 4, torch.bfloat16, 3)
    op = dense_op(x, w, "none", torch.zeros(4, dtype=torch.int64))
    need = lib.tt_dense_workspace_bytes(ctypes.byref(op), 1)
    ws, dw, db = Guarded((1, need), torch.uint8), Guarded((3, 4, 8), torch.bfloat16), Guarded((3, 4), torch.bfloat16)
    assert lib.tt_dense_backward(ctypes.byref(op), None, None, None, None, None, dw.ptr, db.ptr, ws.ptr, need, None) == 0
    assert bool((dw.t == 0).all()) and bool((db.t == 0).all()) and dw.intact() and db.intact()


def test_dense_special_values(lib):
    """Infinities and NaN stay in their rows (in the columns they multiply), and relu passes NaN on."""
    for dtype in DT:
        x, w = torch.ones(5, 8, dtype=dtype), torch.ones(6, 8, dtype=dtype)
        x[1, 3], x[2, 0], x[3, 7] = float("inf"), float("nan"), float("-inf")
        w[4] = 0
        gx, gw, out = place(x), place(w), Guarded((5, 6), dtype)
        for act in ("none", "relu"):
            assert lib.tt_dense_forward(ctypes.byref(dense_op(x, w, act, None)), gx.ptr, gw.ptr, None, None, out.ptr, None, None, 0, None) == 0
            want = ref.act64(x.double() @ w.double().t(), act).to(dtype)
            assert torch.equal(torch.isnan(out.t), torch.isnan(want)) and torch.equal(out.t.nan_to_num(7), want.nan_to_num(7))


def test_dense_half_pre_keeps_the_sign(lib):
    """A pre-activation too small for half precision still has relu's slope of the exact value."""
    x, w = torch.tensor([[2.0 ** -14], [-2.0 ** -14]], dtype=torch.float16), torch.tensor([[2.0 ** -14]], dtype=torch.float16)
    gx, gw, out, pre = place(x), place(w), Guarded((2, 1), torch.float16), Guarded((2, 1), torch.float16)
    assert lib.tt_dense_forward(ctypes.byref(dense_op(x, w, "relu", None)), gx.ptr, gw.ptr, None, None, out.ptr, pre.ptr, None, 0, None) == 0
    assert pre.t[0, 0] > 0 > pre.t[1, 0]


def test_dense_refusals(lib):
    from paper_2507_14668_amd import binding
    x, w, bias, res, grad = make(4, 8, 4, torch.float32)
    offsets = torch.tensor([0, 4])
    gx, gw, out, ws = place(x), place(w), Guarded((4, 4), torch.float32), Guarded((1, 4096), torch.uint8)
    call = lambda op, x=gx.ptr, w=gw.ptr, out=out.ptr, wsp=ws.ptr, size=4096: lib.tt_dense_forward(ctypes.byref(op), x, w, None, None, out, None, wsp, size, None)
    ok = lambda **kw: dense_op(x, w, "relu", None, **kw)
    assert call(ok()) == 0
    assert lib.tt_dense_forward(None, gx.ptr, gw.ptr, None, None, out.ptr, None, ws.ptr, 4096, None) == binding.TT_ERR_INVALID_ARG
    for name, bad, status in (("dtype", 3, -1), ("dtype", -1, -1), ("activation", 5, -1), ("rows", -1, -1), ("rows", 2 ** 31, -2), ("in_dim", 0, -2),
                              ("out_dim", 0, -2), ("in_dim", 2 ** 20 + 1, -2), ("out_dim", 2 ** 20 + 1, -2), ("groups", -1, -1), ("groups", 32769, -2),
                              ("ld_x", 7, -2), ("ld_out", 3, -2), ("ld_residual", 3, -2), ("ld_grad", 3, -2), ("ld_dx", 7, -2), ("ld_x", -8, -2),
                              ("ld_x", 2 ** 41, -2)):
        op = ok()
        setattr(op, name, bad)
        assert call(op) == status, (name, bad)
        assert lib.tt_dense_workspace_bytes(ctypes.byref(op), 1) == 0
    op = ok()
    op.groups = 1  # groups without offsets
    assert call(op) == binding.TT_ERR_INVALID_ARG
    for kw in (dict(x=None), dict(w=None), dict(out=None), dict(x=gx.ptr + 2), dict(w=gw.ptr + 1), dict(out=out.ptr + 2)):
        assert call(ok(), **kw) == binding.TT_ERR_INVALID_ARG, kw
    need = lib.tt_dense_workspace_bytes(ctypes.byref(ok()), 1)
    assert need > 0
    back = lambda pre=gx.ptr, grad=gx.ptr, x=gx.ptr, w=gw.ptr, wsp=ws.ptr, size=need: lib.tt_dense_backward(
        ctypes.byref(ok()), x, w, pre, grad, out.ptr, out.ptr, None, wsp, size, None)
    for kw, status in ((dict(pre=None), -1), (dict(grad=None), -1), (dict(x=None), -1), (dict(w=None), -1), (dict(wsp=None), -3),
                       (dict(size=need - 1), -3), (dict(wsp=ws.ptr + 64), -3)):
        assert back(**kw) == status, kw
    assert lib.tt_dense_backward(ctypes.byref(ok()), None, None, None, None, None, None, None, None, 0, None) == 0  # nothing asked for
    assert offsets.numel() == 2


def matrices(g, out=None, **kw):
    from paper_2507_14668_amd import binding
    m = binding.CMatrices()
    m.dtype, m.batch, m.rows, m.cols = DT[g.dtype], g.shape[0], g.shape[1], g.shape[2]
    for k, v in kw.items():
        setattr(m, k, v)
    return m


def coefs(*c):
    return (ctypes.c_float * len(c))(*c)


@pytest.mark.parametrize("batch,rows,cols,dtype,pad", [(1, 1, 1, torch.float32, 0), (3, 4, 16, torch.float32, 0), (2, 16, 4, torch.bfloat16, 0),
                                                        (2, 33, 70, torch.float32, 3), (1, 70, 33, torch.float16, 1), (5, 1, 9, torch.float32, 0),
                                                        (2, 9, 1, torch.float32, 0), (1, 64, 64, torch.bfloat16, 8),
                                                        (6, 4, 64, torch.float32, 0), (5, 130, 3, torch.float32, 2), (2, 7, 140, torch.bfloat16, 0),
                                                        (1, 300, 8, torch.float16, 0), (1, 3, 512, torch.float32, 0), (2, 9, 260, torch.float32, 1),
                                                        (1, 512, 20, torch.float32, 0), (1, 50, 300, torch.float32, 5), (1, 65, 70, torch.float32, 0),
                                                        (1, 8, 513, torch.float32, 0)])
def test_orthogonalize_values(lib, batch, rows, cols, dtype, pad):
    gen = torch.Generator().manual_seed(rows + cols)
    g = (torch.randn(batch, rows, cols, generator=gen) * 1e-3).to(dtype)
    src = place(g.reshape(batch * rows, cols), cols + pad)
    out = Guarded((batch * rows, cols), dtype, cols + 2 * pad)
    m = matrices(g, row_step=cols + pad, out_row_step=cols + 2 * pad)
    need = lib.tt_orthogonalize_workspace_bytes(ctypes.byref(m))
    ws = Guarded((1, need), torch.uint8)
    assert lib.tt_orthogonalize(ctypes.byref(m), src.ptr, out.ptr, 5, coefs(*(3.4445, -4.7750, 2.0315) * 5), 1e-7, ws.ptr, need, None) == 0
    ref.check_ortho(out.t.reshape(batch, rows, cols), g, "ortho")
    assert src.intact() and out.intact() and ws.intact()
    # in place, other coefficients for each step
    m = matrices(g, row_step=cols + pad, out_row_step=cols + pad)
    steps = ((2.0, -1.5, 0.5), (1.875, -1.25, 0.375))
    assert lib.tt_orthogonalize(ctypes.byref(m), src.ptr, src.ptr, 2, coefs(*sum(steps, ())), 1e-7, ws.ptr, need, None) == 0
    ref.check_ortho(src.t.reshape(batch, rows, cols), g, "ortho in place", steps=2, coefficients=steps)
    assert src.intact()


def test_orthogonalize_special_matrices(lib):
    """Zeros stay zeros, infinities and NaN make their own matrix NaN, sizes near the ends of the range do not matter."""
    gen = torch.Generator().manual_seed(5)
    base = torch.randn(8, 12, generator=gen)
    g = torch.stack([base, torch.zeros(8, 12), base * 1e-25, base * 1e25, base.clone(), base.clone()])
    g[4, 2, 3], g[5, 0, 0] = float("nan"), float("inf")
    src, out = place(g), Guarded((6, 8, 12), torch.float32)
    m = matrices(g)
    need = lib.tt_orthogonalize_workspace_bytes(ctypes.byref(m))
    ws = Guarded((1, need), torch.uint8)
    assert lib.tt_orthogonalize(ctypes.byref(m), src.ptr, out.ptr, 5, coefs(*(3.4445, -4.7750, 2.0315) * 5), 0.0, ws.ptr, need, None) == 0
    ref.check_ortho(out.t[:1], g[:1], "plain", eps=0.0)
    ref.check_ortho(out.t[2:4], g[2:4], "small and large", eps=0.0)
    assert bool(torch.isnan(out.t[4:]).all())
    assert lib.tt_orthogonalize(ctypes.byref(m), src.ptr, out.ptr, 5, coefs(*(3.4445, -4.7750, 2.0315) * 5), 1e-7, ws.ptr, need, None) == 0
    assert bool((out.t[1] == 0).all())


def test_orthogonalize_refusals(lib):
    from paper_2507_14668_amd import binding
    g = torch.randn(2, 4, 4)
    src, ws = place(g), Guarded((1, 65536), torch.uint8)
    c = coefs(*(3.4445, -4.7750, 2.0315) * 5)
    call = lambda m, steps=5, c=c, eps=1e-7, a=src.ptr, b=src.ptr, w=ws.ptr, size=65536: lib.tt_orthogonalize(ctypes.byref(m), a, b, steps, c, eps, w, size, None)
    assert call(matrices(g)) == 0
    for kw in (dict(steps=0), dict(steps=33), dict(c=None), dict(eps=-1.0), dict(eps=float("nan")), dict(a=None), dict(b=None), dict(a=src.ptr + 2),
               dict(c=coefs(*(float("nan"), 0.0, 0.0) * 5))):
        assert call(matrices(g), **kw) == binding.TT_ERR_INVALID_ARG, kw
    for kw in (dict(w=None), dict(size=10), dict(w=ws.ptr + 8)):
        assert call(matrices(g), **kw) == binding.TT_ERR_WORKSPACE, kw
    for kw in (dict(rows=0), dict(cols=0), dict(rows=2 ** 20 + 1), dict(batch=-1), dict(batch=2 ** 33), dict(row_step=3), dict(out_row_step=3),
               dict(out_batch_step=5), dict(batch_step=-1)):
        assert call(matrices(g, **kw)) == binding.TT_ERR_SHAPE, kw
    assert call(matrices(g, dtype=3)) == binding.TT_ERR_INVALID_ARG
    assert call(matrices(g, batch=0), a=None, b=None) == 0
    assert lib.tt_orthogonalize_workspace_bytes(ctypes.byref(matrices(g, rows=0))) == 0


def core_case(n, d, R, seed):
    gen = torch.Generator().manual_seed(seed)
    r = (1, R[0], R[1], 1)
    numel = [r[k] * n[k] * d[k] * r[k + 1] for k in range(3)]
    mk = lambda std: [torch.randn(x, generator=gen) * std for x in numel]
    return r, mk(0.05), mk(1e-3), mk(1e-2)


def core_update64(n, d, r, cores, grads, momenta, lr, mu, nesterov, **how):
    """New cores and momenta in 64 bits, and the slices' updates u with the orthogonalised ones."""
    new, mom, us = [], [], []
    for k in range(3):
        m = mu * momenta[k].double() + grads[k].double()
        u = grads[k].double() + mu * m if nesterov else m
        rows, cols = (d[0], r[1]) if k == 0 else (r[k], d[k] * r[k + 1])
        view = lambda t: t.view(r[k], n[k], -1).permute(1, 0, 2).reshape(n[k], rows, cols)
        o = ref.ortho(view(u), **how)
        back = o.reshape(n[k], r[k], -1).permute(1, 0, 2).reshape(-1)
        new.append(cores[k].double() - lr * max(1.0, rows / cols) ** 0.5 * back)
        mom.append(m)
        us.append(view(u))
    return new, mom, us


@pytest.mark.parametrize("n,d,R,nesterov", [((3, 5, 2), (2, 2, 4), (4, 4), 1), ((2, 3, 4), (4, 2, 3), (5, 7), 0), ((1, 2, 1), (1, 1, 1), (1, 1), 1)])
def test_core_update_values(lib, n, d, R, nesterov):
    from paper_2507_14668_amd import binding
    r, cores, grads, momenta = core_case(n, d, R, 3)
    grads[1].view(r[1], n[1], -1)[:, 0] = 0
    momenta[1].view(r[1], n[1], -1)[:, 0] = 0  # a slice that nothing touched
    t = binding.CTable()
    t.num_rows, t.n[:], t.d[:], t.r[:] = n[0] * n[1] * n[2], n, d, r
    hold = [[place(x[None]) for x in xs] for xs in (cores, grads, momenta)]
    for k in range(3):
        t.core[k] = hold[0][k].ptr
    arr = lambda gs: (ctypes.c_void_p * 3)(*[g.ptr for g in gs])
    need = lib.tt_core_ortho_workspace_bytes(ctypes.byref(t))
    ws = Guarded((1, need), torch.uint8)
    c = coefs(*(3.4445, -4.7750, 2.0315) * 5)
    call = lambda w=ws.ptr, size=need, steps=5, m=None: lib.tt_core_ortho_update(ctypes.byref(t), arr(hold[1]), m or arr(hold[2]), 0.02, 0.9, nesterov, steps, c,
                                                                                  1e-7, w, size, None)
    assert call(size=need - 1) == binding.TT_ERR_WORKSPACE and call(w=None) == binding.TT_ERR_WORKSPACE
    assert call(steps=0) == binding.TT_ERR_INVALID_ARG and call(m=(ctypes.c_void_p * 3)(None, None, None)) == binding.TT_ERR_INVALID_ARG
    assert call() == 0
    new, mom, us = core_update64(n, d, r, cores, grads, momenta, 0.02, 0.9, nesterov)
    for k in range(3):
        # each update is off by at most 3 times what the formula in fp32 is off, times lr and the slices' factor; the momentum and
        # the step are rounded once or twice each
        off = (ref.ortho(us[k].float(), dtype=torch.float32).double() - ref.ortho(us[k])).norm()
        err = (hold[0][k].t[0].double() - new[k]).norm()
        assert err <= 0.02 * 4 * (3 * off + 16 * ref.U * ref.ortho(us[k]).norm()) + 2 * ref.U * new[k].norm(), k
        ref.check(hold[2][k].t[0], mom[k], 3 * ref.U * (mom[k].abs() + momenta[k].abs()), "momentum %d" % k)
        for side in hold:
            assert side[k].intact()
    assert torch.equal(hold[0][1].t[0].view(r[1], n[1], -1)[:, 0], cores[1].view(r[1], n[1], -1)[:, 0])
    assert ws.intact()
    t.r[1] = 129
    assert lib.tt_core_ortho_workspace_bytes(ctypes.byref(t)) == 0 and call() == binding.TT_ERR_SHAPE


@pytest.mark.parametrize("rows,k,n,groups", [(1, 8, 1, 0), (70, 64, 66, 0), (33, 21, 40, 0), (40, 600, 40, 0), (130, 48, 130, 0), (90, 64, 70, 3)])
def test_relu_decides_the_sign_exactly(lib, rows, k, n, groups):
    """fp32 relu: biases that cancel a column's sum for one row down to its last bits, so that fp32 sums have any sign: the stored
    pre-activation is the exact value's, to half a step of it and 64-bit rounding of the terms."""
    x, w, _, _, grad = make(rows, k, n, torch.float32, groups, seed=rows + k)
    offsets = torch.tensor([0, 25, 25, 80]) if groups else None
    where = [(min(c, rows - 1), c, 0) for c in range(n)]  # the row that each column's bias cancels, and its group
    if groups:
        where = [(lo + c % (hi - lo), c, g) for g, (lo, hi) in enumerate(ref.ranges(offsets, 3, rows)) if hi > lo for c in range(n)]
    bias = torch.zeros(w.shape[:-1])
    exact = {}
    for m, c, g in where:
        wg, bg = (w[g], bias[g]) if groups else (w, bias)
        s = float((x[m].double() * wg[c].double()).sum())
        bg[c] = -s
        exact[m, c] = s + float(bg[c]), float((x[m].double() * wg[c].double()).abs().sum())
    gx, gw, gb, out, pre = place(x), place(w), place(bias), Guarded((rows, n), torch.float32), Guarded((rows, n), torch.float32)
    op = dense_op(x, w, "relu", offsets)
    need = lib.tt_dense_workspace_bytes(ctypes.byref(op), 0)
    ws = Guarded((1, max(1, need)), torch.uint8)
    assert lib.tt_dense_forward(ctypes.byref(op), gx.ptr, gw.ptr, gb.ptr, None, out.ptr, pre.ptr, ws.ptr, need, None) == 0
    assert any(z != 0 for z, _ in exact.values())
    for (m, c), (z, size) in exact.items():
        got = float(pre.t[m, c])
        assert abs(got - z) <= ref.U * abs(z) + 2 * k * 2.0 ** -53 * size, (m, c, got, z)
        if abs(z) > 2 * k * 2.0 ** -53 * size:
            assert (got > 0) == (z > 0) and (float(out.t[m, c]) > 0) == (z > 0), (m, c, got, z)
    want, tol, z, tz = ref.forward64(x, w, bias, None, "relu", offsets)
    member = ~torch.isnan(z[:, 0])
    ref.check(out.t[member], want[member], tol[member], "out")
    ref.check(pre.t[member], z[member], tz[member], "pre")
    for g in (gx, gw, gb, out, pre, ws):
        assert g.intact()


@pytest.mark.parametrize("dtype", DT, ids=str)
@pytest.mark.parametrize("offs", [None, [0, 20, 64], [0, 64, 64]])
def test_bias_gradient_beside_special_values(lib, dtype, offs):
    """A NaN or an infinity in a column of the gradient reaches that column's sum only, with and without the weights' gradient beside it, and the
    other sums have the bits that they have without it (fp32: they may be formed by another instruction then)."""
    rows, k, n = 64, 264, 264
    groups = 0 if offs is None else len(offs) - 1
    offsets = None if offs is None else torch.tensor(offs, dtype=torch.int64)
    x, w, _, _, grad = make(rows, k, n, dtype, groups)
    op = dense_op(x, w, "none", offsets)
    need = lib.tt_dense_workspace_bytes(ctypes.byref(op), 1)
    gx, ws = place(x), Guarded((1, need), torch.uint8)

    def dbias(g, with_dw):
        gg, ow, ob = place(g), Guarded(tuple(w.shape), dtype), Guarded(tuple(w.shape[:-1]), dtype)
        assert lib.tt_dense_backward(ctypes.byref(op), gx.ptr, None, None, gg.ptr, None, ow.ptr if with_dw else None, ob.ptr, ws.ptr, need, None) == 0
        assert ow.intact() and ob.intact() and ws.intact()
        return ob.t.clone().view(-1, n)
    clean = dbias(grad, True)
    # fp32 sums of m terms are each within 2 (m + 2) u sum |terms| of the exact one, so two of them within twice that of each other
    most = 0.0 if dtype != torch.float32 else 4 * (rows + 2) * ref.U * float(grad.double().abs().sum(0).max())
    assert torch.equal(dbias(grad, False), clean)
    for value, cols in ((float("nan"), (7,)), (float("inf"), (7,)), (float("-inf"), (130, 263)), (float("inf"), (0, 16))):
        bad = grad.clone()
        bad[rows - 1, list(cols)] = value
        want = clean.clone()
        member = [(lo, hi) for lo, hi in ref.ranges(offsets, max(groups, 1), rows)]
        for g, (lo, hi) in enumerate(member):
            if lo <= rows - 1 < hi:
                want[g, list(cols)] = value
        for with_dw in (True, False):
            got = dbias(bad, with_dw)
            assert torch.equal(got.isnan(), want.isnan()), (value, cols, with_dw)
            off = (got.nan_to_num(3.0, 4.0, 5.0).double() - want.nan_to_num(3.0, 4.0, 5.0).double()).abs()
            assert bool((off <= most).all()), (value, cols, with_dw)


@pytest.mark.parametrize("small,large", [(2.0 ** -115, 2.0 ** 105), (1e-35, 1e20), (2e-38, 1e25), (1e-36, 1.0), (3e-32, 1e38), (1e-30, 1e-6), (2.0 ** -90, 2.0 ** 3)])
@pytest.mark.parametrize("rows,k,n", [(40, 32, 40), (70, 300, 66)])
def test_small_numbers_beside_large_ones(lib, small, large, rows, k, n):
    """Normal fp32 numbers near the lower end, in all of one operand or in a single entry of it, keep their 24 bits whatever they are multiplied by:
    within 2 (K + 2) u sum |terms|, as everywhere."""
    x, w, _, _, grad = make(rows, k, n, torch.float32, seed=3)
    one = lambda t: torch.where(t == 0, torch.ones(()), t)
    for a, b in ((small * one(x), large * one(w)), (large * one(x), small * one(w))):
        for single in (False, True):
            if single:  # one small number in each row (each column of the weight's), beside ones that sum to nothing
                a, b = a.clone(), b.clone()
                t = a if small * 100 > float(a.abs().max()) else b
                keep = torch.zeros_like(t)
                keep[torch.arange(t.shape[0]), torch.arange(t.shape[0]) % k] = 1.0
                t.mul_(keep)
            ga, gb, out = place(a), place(b), Guarded((rows, n), torch.float32)
            op = dense_op(a, b, "none", None)
            need = lib.tt_dense_workspace_bytes(ctypes.byref(op), 0)
            ws = Guarded((1, max(1, need)), torch.uint8)
            assert lib.tt_dense_forward(ctypes.byref(op), ga.ptr, gb.ptr, None, None, out.ptr, None, ws.ptr, need, None) == 0
            want, size = a.double() @ b.double().t(), a.double().abs() @ b.double().abs().t()
            # (and half of the smallest number for each term, where results are that small)
            fine = torch.isfinite(size)  # (1e38 times three and more is an infinity: those rows have infinities and NaN where the formula has them)
            ref.check(out.t[fine], want[fine], (2 * (k + 2) * ref.U * size + (k + 1) * 2.0 ** -149)[fine], "small beside large")
            assert torch.equal(out.t[~fine].double().nan_to_num(7.0), want[~fine].nan_to_num(7.0))
            assert out.intact() and ws.intact()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
def test_gelu_of_16_bits_over_its_tail(lib, dtype):
    """Value and slope to half a step of the type, relative to themselves, down to where they leave its range."""
    z = torch.arange(-2 ** 15, 2 ** 15, dtype=torch.int32).to(torch.int16).view(dtype)
    z = z[torch.isfinite(z) & (z >= -12.75) & (z <= 8) & (z.float().abs() >= 2.0 ** -8)][::7]
    # Phi to 2e-6, the rounding of z^2 / 2 and of exp's argument, a few units for the rest; then half a step of the type
    z64 = z.double()
    phi, bell = 0.5 * torch.erfc(-z64 / math.sqrt(2)), torch.exp(-0.5 * z64 * z64) / math.sqrt(2 * math.pi)
    near = 2e-6 + (z64 * z64 + 8) * ref.U
    gx, gw, out, one, dx = place(z[:, None]), place(torch.ones(1, 1, dtype=dtype)), Guarded((len(z), 1), dtype), place(torch.ones(len(z), 1, dtype=dtype)), Guarded((len(z), 1), dtype)
    op = dense_op(gx.t, gw.t, "gelu", None)
    need = lib.tt_dense_workspace_bytes(ctypes.byref(op), 1)
    ws = Guarded((1, need), torch.uint8)
    assert lib.tt_dense_forward(ctypes.byref(op), gx.ptr, gw.ptr, None, None, out.ptr, None, ws.ptr, need, None) == 0
    want = z64 * phi
    ref.check(out.t[:, 0], want, near * want.abs() + ref.rounding(want, dtype), "gelu")
    assert lib.tt_dense_backward(ctypes.byref(op), gx.ptr, gw.ptr, gx.ptr, one.ptr, dx.ptr, None, None, ws.ptr, need, None) == 0
    want = phi + z64 * bell
    ref.check(dx.t[:, 0], want, near * (phi + z64.abs() * bell) + ref.rounding(want, dtype), "slope")


def test_outputs_over_inputs_are_refused(lib):
    """Workgroups read what others have written by then: no output starts where an input does, but for the residual's own rows."""
    from paper_2507_14668_amd import binding
    x, w, bias, res, _ = make(4, 4, 4, torch.float32)
    gx, gw, gb, gr, out, pre, ws = place(x), place(w), place(bias), place(res), Guarded((4, 4), torch.float32), Guarded((4, 4), torch.float32), Guarded((1, 8192), torch.uint8)
    f = lambda op, out, pre=None, res=gr.ptr: lib.tt_dense_forward(ctypes.byref(op), gx.ptr, gw.ptr, gb.ptr, res, out, pre, ws.ptr, 8192, None)
    op = dense_op(x, w, "relu", None)
    bad = binding.TT_ERR_INVALID_ARG
    assert [f(op, o.ptr) for o in (gx, gw, gb)] == [bad] * 3 and [f(op, out.ptr, p.ptr) for p in (gx, gw, gb, gr, out)] == [bad] * 5
    assert f(op, gr.ptr, pre.ptr) == 0 and f(op, out.ptr) == 0 and f(op, out.ptr, pre.ptr, None) == 0
    assert f(dense_op(x, w, "relu", None, ld_out=8, ld_residual=4), gr.ptr) == bad
    gg = place(res)
    b = lambda dx, dw, db: lib.tt_dense_backward(ctypes.byref(op), gx.ptr, gw.ptr, pre.ptr, gg.ptr, dx, dw, db, ws.ptr, 8192, None)
    for t in (gx, gw, pre, gg):
        assert b(t.ptr, None, None) == bad and b(None, t.ptr, None) == bad and b(None, None, t.ptr) == bad
    assert b(out.ptr, None, None) == 0
    g = torch.randn(2, 4, 4)
    src, c = place(g), coefs(*(3.4445, -4.7750, 2.0315) * 5)
    ortho = lambda m: lib.tt_orthogonalize(ctypes.byref(m), src.ptr, src.ptr, 5, c, 1e-7, ws.ptr, 8192, None)
    assert ortho(matrices(g, batch=1, row_step=8)) == bad and ortho(matrices(g, batch_step=8, out_batch_step=16, row_step=4)) == bad
    assert ortho(matrices(g)) == 0
    for t in (gx, gw, gb, gr, out, pre, ws, gg, src):
        assert t.intact()
