"""The dense operators on the GPU: values against 64 bits over sizes, types, layouts and groups; autograd, the modules that call
them, streams, graphs, reproducibility and refusals."""
import math

import pytest
import torch

import dense_ref as ref

pytestmark = pytest.mark.gpu
DTYPES = (torch.float32, torch.bfloat16, torch.float16)


@pytest.fixture(scope="module")
def tt():
    import paper_2507_14668_amd as tt
    return tt


def make(rows, k, n, dtype, groups=0, seed=0, pad=0, shift=0):
    """CUDA inputs; with `pad` rows are views into wider ones, with `shift` nothing is aligned to more than an element."""
    gen = torch.Generator().manual_seed(seed)
    lead = (groups,) if groups else ()

    def f(*s, std=1.0, pad=0):
        wide = torch.zeros(*s[:-1], s[-1] + pad, dtype=dtype)
        flat = torch.empty(wide.numel() + shift, dtype=dtype, device="cuda")[shift:].view(wide.shape)
        t = flat[..., :s[-1]]
        t.copy_((torch.randn(*s, generator=gen) * std).to(dtype))
        return t
    return f(rows, k, pad=pad), f(*lead, n, k, std=k ** -0.5), f(*lead, n), f(rows, n, pad=pad), f(rows, n, pad=pad)


def cpu(*ts):
    return [None if t is None else t.detach().cpu() for t in ts]


def offsets_of(sizes, first=0):
    return torch.tensor([first] + list(sizes), dtype=torch.int64).cumsum(0)


SIZES = [
    # rows, k, n, group sizes (None: one weight), pad, shift
    (1, 1, 1, None, 0, 0),
    (1, 128, 512, None, 0, 0),
    (1, 4096, 130, None, 0, 0),
    (1, 37, 4097, None, 0, 1),
    (2, 264, 520, None, 0, 0),
    (5, 1000, 96, None, 0, 0),
    (16, 512, 640, None, 0, 0),
    (17, 520, 250, None, 8, 0),
    (33, 2050, 66, None, 0, 0),
    (64, 1024, 1024, None, 0, 0),
    (65, 63, 65, None, 1, 1),
    (127, 129, 255, None, 0, 3),
    (128, 128, 128, None, 0, 0),
    (256, 64, 256, None, 0, 0),
    (300, 72, 264, None, 8, 0),
    (257, 320, 512, None, 0, 0),
    (700, 512, 768, None, 64, 0),
    (1000, 479, 513, None, 5, 0),
    (2048, 1024, 256, None, 0, 0),
    (4097, 136, 384, None, 0, 0),
    (5000, 16, 24, None, 0, 0),
    (2050, 200, 2100, None, 0, 0),
    (2100, 131, 2049, None, 3, 1),
    (8200, 2056, 520, None, 8, 0),
    (6000, 96, 700, (2500, 0, 1, 3499), 0, 0),
    (5000, 328, 1030, (130, 2700, 5, 2100), 6, 0),
    (4100, 136, 2600, None, 8, 0),    # the largest tiles: forward, gradient of x, gradient of w
    (4100, 2600, 200, None, 8, 0),
    (300, 4096, 2568, None, 0, 0),
    (12000, 1024, 1024, (9300, 0, 3, 257, 1000, 64, 700, 128, 300, 1, 100, 147), 0, 0),
    (9000, 64, 40, (8000, 10, 990), 0, 0),
    (9000, 33, 47, (10, 8000, 0, 990), 1, 1),
    (30, 128, 512, (3, 0, 1, 26), 0, 0),
    (100, 64, 72, (1,) * 100, 0, 0),
    (515, 128, 128, (0, 256, 0, 1, 258, 0), 0, 0),
    (1500, 256, 320, (700, 0, 90, 710), 8, 0),
    (900, 77, 131, (300, 299, 301), 3, 1),
    (2000, 512, 512, (1900, 100), 0, 0),
    (400, 40, 48, tuple([2, 0, 4] * 65), 0, 0),
]


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("rows,k,n,sizes,pad,shift", SIZES)
def test_values(tt, rows, k, n, sizes, pad, shift, dtype):
    act = ref.ACTS[(rows + k + n) % 5]
    extras = (rows + n) % 3 != 0
    groups = 0 if sizes is None else len(sizes)
    x, w, bias, res, grad = make(rows, k, n, dtype, groups, seed=rows + n, pad=pad, shift=shift)
    if not extras:
        bias = res = None
    off = None if sizes is None else offsets_of(sizes)
    doff = None if off is None else off.cuda()
    pre = torch.full((rows, n), math.nan, dtype=dtype, device="cuda")
    out = tt.tt_dense_forward(x, w, bias, res, act, offsets=doff, pre=pre)
    want, tol, z, tz = ref.forward64(*cpu(x, w, bias, res), act, off)
    member = ~torch.isnan(z[:, 0])
    got, gpre = cpu(out, pre)
    ref.check(got[member], want[member], tol[member], "out")
    ref.check(gpre[member], z[member], tz[member], "pre")
    assert bool((got[~member] == 0).all())
    pz = z.nan_to_num(0).to(dtype)
    (dx, dw, db), (tx, tw, tb) = ref.backward64(*cpu(x, w, grad), pz, act, off)
    dpz = pz.cuda()
    gx, gw, gb = cpu(*tt.tt_dense_backward(x, w, grad, dpz, act, offsets=doff))
    ref.check(gx[member], dx[member], tx[member], "dx")
    assert bool((gx[~member] == 0).all())
    ref.check(gw, dw, tw, "dw")
    ref.check(gb, db, tb, "dbias")
    # each of them alone, and the same bits again
    for i in range(3):
        alone = tt.tt_dense_backward(x, w, grad, dpz, act, offsets=doff, needs=tuple(j == i for j in range(3)))
        assert [t is None for t in alone] == [j != i for j in range(3)]
        assert torch.equal(alone[i].cpu(), (gx, gw, gb)[i]), "gradient %d by itself" % i
    again = tt.tt_dense_forward(x, w, bias, res, act, offsets=doff)
    assert torch.equal(again, out)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("act", ref.ACTS)
def test_every_activation(tt, act, dtype):
    """Steep and flat parts, both ends: z from -40 to 40, and infinities."""
    z = torch.cat([torch.linspace(-40, 40, 4001), torch.linspace(-1, 1, 999), torch.tensor([0.0, -0.0, 1e-6, -1e-6])]).to(dtype)
    x, w = z[:, None].cuda(), torch.ones(1, 1, dtype=dtype, device="cuda")
    want, tol, _, _ = ref.forward64(z[:, None], w.cpu(), None, None, act)
    ref.check(tt.tt_dense_forward(x, w, activation=act).cpu(), want, tol, act)
    grad = torch.ones_like(x)
    (dx, _, _), (tx, _, _) = ref.backward64(z[:, None], w.cpu(), grad.cpu(), z[:, None], act)
    ref.check(tt.tt_dense_backward(x, w, grad, x.contiguous(), act, needs=(True, False, False))[0].cpu(), dx, tx, act + " slope")
    ends = torch.tensor([[math.inf], [-math.inf]], dtype=dtype, device="cuda")
    slope = tt.tt_dense_backward(ends, w, torch.ones_like(ends), ends, act, needs=(True, False, False))[0].cpu().flatten().tolist()
    assert slope == {"none": [1, 1], "relu": [1, 0], "gelu": [1, 0], "silu": [1, 0], "sigmoid": [0, 0]}[act]


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("rows,k,n", [(3, 64, 96), (40, 264, 128), (300, 512, 520)])
def test_special_values_stay_in_their_rows(tt, rows, k, n, dtype):
    x, w, bias, _, _ = make(rows, k, n, dtype)
    x[0, k - 1], x[1, 0], x[2, 5] = math.inf, math.nan, -math.inf
    for act in ("none", "relu"):
        out = tt.tt_dense_forward(x, w, bias, None, act).cpu()
        want, tol, _, _ = ref.forward64(*cpu(x, w, bias), None, act)
        for r in (0, 1, 2):
            assert torch.equal(torch.isnan(out[r]), torch.isnan(want[r])), r
            fine = ~torch.isnan(want[r])
            assert torch.equal(out[r][fine].double(), want[r][fine]), r
        ref.check(out[3:], want[3:], tol[3:], "the other rows")
    # a NaN in one column of the gradient reaches that column of x's weights only
    grad = torch.ones(rows, n, dtype=dtype, device="cuda")
    grad[rows - 1, 7] = math.nan
    good = torch.ones(rows, k, dtype=dtype, device="cuda")
    dx, dw, db = tt.tt_dense_backward(good, w, grad)
    assert bool(torch.isnan(dx[rows - 1]).all()) and not bool(torch.isnan(dx[:rows - 1]).any())
    assert bool(torch.isnan(dw[7]).all()) and int(torch.isnan(dw).any(1).sum()) == 1
    assert bool(torch.isnan(db[7])) and int(torch.isnan(db).sum()) == 1


@pytest.mark.parametrize("scale", [1e-30, 1e-18, 1e18, 3e38])
def test_float32_over_its_range(tt, scale):
    """Products of numbers near both ends: infinities where 32 bits have them, no loss of precision before."""
    for rows, k, n in ((8, 64, 96), (300, 256, 512)):
        x, w, _, _, _ = make(rows, k, n, torch.float32)
        x = x / x.abs().max() * scale
        for factor in (1.0, 1e-6 if scale > 1 else 1e6):
            wf = w * factor
            out = tt.tt_dense_forward(x, wf).cpu()
            want, tol, _, _ = ref.forward64(*cpu(x, wf))
            over = want.abs() > 3.4e38
            near = (want.abs() + tol > 3.3e38) & ~over
            size = x.cpu().double().abs() @ wf.cpu().double().abs().t()
            fine = ~over & ~near & (size < 3e38)
            ref.check(torch.where(fine, out, torch.zeros(())), torch.where(fine, want, torch.zeros((), dtype=torch.float64)),
                      torch.where(fine, tol, torch.zeros((), dtype=torch.float64)) + 1e-300 + k * 2.0 ** -149, "scale %g" % scale)


@pytest.mark.parametrize("offs", [[3, 40, 60], [0, 50, 20, 64], [-9, 10, 400], [64, 64, 64], [90, 95], [0, 0, 0, 64]])
def test_offsets_of_any_kind(tt, offs):
    """Rows outside every group, offsets that fall, leave the rows, or cover nothing."""
    off = torch.tensor(offs)
    x, w, bias, res, grad = make(64, 40, 72, torch.bfloat16, len(offs) - 1)
    out = torch.full((64, 72), 5.0, dtype=torch.bfloat16, device="cuda")
    pre = torch.full((64, 72), 6.0, dtype=torch.bfloat16, device="cuda")
    tt.tt_dense_forward(x, w, bias, res, "gelu", offsets=off.cuda(), out=out, pre=pre)
    want, tol, z, tz = ref.forward64(*cpu(x, w, bias, res), "gelu", off)
    member = ~torch.isnan(z[:, 0])
    ref.check(out.cpu()[member], want[member], tol[member], "out")
    ref.check(pre.cpu()[member], z[member], tz[member], "pre")
    assert bool((out.cpu()[~member] == 5).all()) and bool((pre.cpu()[~member] == 6).all())
    pz = z.nan_to_num(0).bfloat16()
    (dx, dw, db), (tx, tw, tb) = ref.backward64(*cpu(x, w, grad), pz, "gelu", off)
    grad[~member.cuda()] = math.nan  # rows of no group reach nothing
    gx, gw, gb = cpu(*tt.tt_dense_backward(x, w, grad, pz.cuda(), "gelu", offsets=off.cuda()))
    ref.check(gx[member], dx[member], tx[member], "dx")
    assert bool((gx[~member] == 0).all())
    ref.check(gw, dw, tw, "dw")
    ref.check(gb, db, tb, "dbias")


def test_no_rows(tt):
    x, w, bias, _, _ = make(0, 16, 8, torch.float32)
    assert tt.tt_dense_forward(x, w, bias).shape == (0, 8)
    dx, dw, db = tt.tt_dense_backward(x, w, torch.empty(0, 8, device="cuda"))
    assert dx.shape == (0, 16) and bool((dw == 0).all()) and bool((db == 0).all())


def test_residual_in_place_and_row_views(tt):
    x, w, bias, res, _ = make(200, 96, 160, torch.bfloat16, pad=16)
    want = tt.tt_dense_forward(x, w, bias, res, "silu")
    base = torch.full((200, 176), 3.0, dtype=torch.bfloat16, device="cuda")
    view = base[:, 8:168]
    view.copy_(res)
    got = tt.tt_dense_forward(x, w, bias, view, "silu", out=view)
    assert got.data_ptr() == view.data_ptr() and torch.equal(view, want)
    assert bool((base[:, :8] == 3).all()) and bool((base[:, 168:] == 3).all())


@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("act", ref.ACTS)
def test_autograd_against_formula_and_differences(tt, act, grouped):
    """The gradients of the autograd call are those of the formula, and those of differences of the 64-bit forward."""
    rows, k, n = 37, 24, 20
    off = torch.tensor([0, 12, 12, 37]) if grouped else None
    x, w, bias, res, grad = make(rows, k, n, torch.float32, 3 if grouped else 0)
    leaves = [t.detach().contiguous().requires_grad_(True) for t in (x, w, bias, res)]
    out = tt.tt_dense(*leaves, act, offsets=None if off is None else off.cuda())
    got = [g.cpu().double() for g in torch.autograd.grad(out, leaves, grad)]
    cx, cw, cb, cr, cg = cpu(x, w, bias, res, grad)
    _, _, z, _ = ref.forward64(cx, cw, cb, cr, act, off)
    (dx, dw, db), (tx, tw, tb) = ref.backward64(cx, cw, cg, z.float(), act, off)
    for g, want, tol, name in zip(got, (dx, dw, db), (tx, tw, tb), ("dx", "dw", "dbias")):
        # z is the kernel's own: at most its error away, times the slope's slope (at most 0.8)
        ref.check(g, want, tol + 1e-5 * want.abs().max(), name)
    assert torch.equal(got[3].float(), cg)
    # differences of the loss <out, grad> along a random direction, in 64 bits
    gen = torch.Generator().manual_seed(9)
    if act != "relu":  # (a kink makes differences wrong)
        h = 1e-5
        loss = lambda ts: float((ref.forward64(*ts, act, off)[0] * cg.double()).sum())
        for i, t in enumerate((cx, cw, cb, cr)):
            way = torch.randn(t.shape, generator=gen, dtype=torch.float64)
            sides = []
            for s in (h, -h):
                args = [a.double() for a in (cx, cw, cb, cr)]
                args[i] = args[i] + s * way
                sides.append(_loss64(args, act, off, cg))
            slope = (sides[0] - sides[1]) / (2 * h)
            mine = float((got[i] * way).sum())
            # h^2 / 6 of the third derivative and 2^-52 / h of the loss; the gradients' own 1e-5
            assert abs(mine - slope) <= 2e-5 * float((got[i].abs() * way.abs()).sum()) + 1e-6, (i, mine, slope)
        assert loss((cx, cw, cb, cr)) == loss((cx, cw, cb, cr))


def _loss64(args, act, off, grad):
    x, w, b, r = args
    ws, bs = (w, b) if off is not None else (w[None], b[None])
    total = 0.0
    for g, (lo, hi) in enumerate(ref.ranges(off, ws.shape[0], x.shape[0])):
        y = ref.act64(x[lo:hi] @ ws[g].t() + bs[g], act) + r[lo:hi]
        total += float((y * grad[lo:hi].double()).sum())
    return total


def test_autograd_takes_expanded_gradients_and_frozen_inputs(tt):
    x, w, bias, res, _ = make(50, 32, 24, torch.bfloat16)
    leaves = [t.detach().clone().requires_grad_(True) for t in (x, w, bias, res)]
    grads = torch.autograd.grad(tt.tt_dense(*leaves, "silu").sum(), leaves)   # a gradient with steps of zero
    ones = torch.ones(50, 24, dtype=torch.bfloat16, device="cuda")
    want = torch.autograd.grad(tt.tt_dense(*leaves, "silu"), leaves, ones)
    assert all(torch.equal(a, b) for a, b in zip(grads, want))
    for i in range(4):
        part = [t.detach().requires_grad_(j == i) for j, t in enumerate(leaves)]
        (g,) = torch.autograd.grad(tt.tt_dense(*part, "silu"), part[i], ones)
        assert torch.equal(g, want[i]), i
    strided = x.t().contiguous().t().detach().requires_grad_(True)  # columns apart: copied within the call
    (g,) = torch.autograd.grad(tt.tt_dense(strided, w), strided, ones)
    assert torch.equal(g, torch.autograd.grad(tt.tt_dense(leaves[0], w), leaves[0], ones)[0])


def test_residual_gradient_outside_groups_is_zero(tt):
    x, w, bias, res, grad = make(30, 16, 8, torch.float32, 2)
    res = res.detach().requires_grad_(True)
    out = tt.tt_dense(x, w, bias, res, offsets=torch.tensor([4, 10, 25], device="cuda"))
    (g,) = torch.autograd.grad(out, res, grad)
    assert bool((g[:4] == 0).all()) and bool((g[25:] == 0).all()) and torch.equal(g[4:25], grad[4:25])
    assert bool((out[:4] == 0).all()) and bool((out[25:] == 0).all())


def test_streams_graphs_and_overlapping_calls(tt):
    """A call on a stream of its own, two at once, and a captured training pass replayed over new inputs with eager work between."""
    x, w, bias, res, grad = make(777, 256, 320, torch.bfloat16, 3)
    off = torch.tensor([0, 300, 300, 777], device="cuda")
    want = tt.tt_dense_forward(x, w, bias, res, "gelu", offsets=off)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for s in streams:
        outs.append(tt.tt_dense_forward(x, w, bias, res, "gelu", offsets=off, stream=s))
    for s in streams:
        s.synchronize()
    assert all(torch.equal(o, want) for o in outs)

    def step():
        pre = torch.empty(777, 320, dtype=torch.bfloat16, device="cuda")
        out = tt.tt_dense_forward(x, w, bias, res, "gelu", offsets=off, pre=pre)
        return (out,) + tt.tt_dense_backward(x, w, grad, pre, "gelu", offsets=off)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        gen = torch.Generator(device="cuda").manual_seed(i)
        x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        off.copy_(torch.tensor([0, 100 * i, 100 * i + 7, 777 - i], device="cuda"))
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), i


def test_refusals(tt):
    x, w, bias, res, grad = make(10, 16, 8, torch.float32)
    off = torch.tensor([0, 10], device="cuda")
    for error, call in (
            (TypeError, lambda: tt.tt_dense_forward(x.cpu(), w)),
            (TypeError, lambda: tt.tt_dense_forward(x.double(), w.double())),
            (TypeError, lambda: tt.tt_dense_forward(x, w.bfloat16())),
            (TypeError, lambda: tt.tt_dense_forward(x, w, bias.half())),
            (TypeError, lambda: tt.tt_dense_forward(x, w, None, res.half())),
            (TypeError, lambda: tt.tt_dense_forward(x, w.t().contiguous().t())),
            (TypeError, lambda: tt.tt_dense_forward(x, w[None], offsets=off.int())),
            (ValueError, lambda: tt.tt_dense_forward(x, w[None])),
            (ValueError, lambda: tt.tt_dense_forward(x, w, offsets=off)),
            (ValueError, lambda: tt.tt_dense_forward(x, w[None], offsets=torch.zeros(3, dtype=torch.int64, device="cuda"))),
            (ValueError, lambda: tt.tt_dense_forward(x[:, :8], w)),
            (ValueError, lambda: tt.tt_dense_forward(x, w, bias[:4].contiguous())),
            (ValueError, lambda: tt.tt_dense_forward(x, w, None, res[:5])),
            (ValueError, lambda: tt.tt_dense_forward(x, w, activation="tanh")),
            (ValueError, lambda: tt.tt_dense_forward(x, w, out=torch.empty(10, 9, device="cuda"))),
            (ValueError, lambda: tt.tt_dense_forward(x.t().contiguous().t(), w)),
            (ValueError, lambda: tt.tt_dense_forward(x[:1].expand(10, 16), w)),
            (ValueError, lambda: tt.tt_dense_backward(x, w, grad, activation="relu")),
            (ValueError, lambda: tt.tt_dense_backward(x, w, grad[:, :4])),
            (TypeError, lambda: tt.tt_orthogonalize(w.cpu())),
            (TypeError, lambda: tt.tt_orthogonalize(w.double())),
            (ValueError, lambda: tt.tt_orthogonalize(w[0])),
            (ValueError, lambda: tt.tt_orthogonalize(w.t())),
            (ValueError, lambda: tt.tt_orthogonalize(w, steps=0)),
            (ValueError, lambda: tt.tt_orthogonalize(w, coefficients=((1, 2, 3), (1, 2, 3)))),
            (ValueError, lambda: tt.tt_orthogonalize(w, out=w[:4])),
            (tt.TTError, lambda: tt.tt_orthogonalize(w, eps=-1.0)),
            (tt.TTError, lambda: tt.tt_orthogonalize(w, workspace=torch.empty(128, dtype=torch.uint8, device="cuda"))),
            (tt.TTError, lambda: tt.tt_dense_backward(x, w, grad, x[:, :8].contiguous(), "silu", workspace=torch.empty(0, dtype=torch.uint8, device="cuda")))):
        with pytest.raises(error):
            call()
    torch.cuda.synchronize()


# ---- orthogonalised updates ------------------------------------------------------------------------
ORTHO = [(1, 1, 1), (3, 1, 40), (2, 40, 1), (7, 4, 64), (7, 64, 4), (2, 64, 512), (1, 512, 128), (3, 100, 260), (1, 129, 129), (2, 128, 700), (1, 300, 290),
         (1, 700, 333), (40, 33, 17), (1, 16, 3000), (1, 2500, 24), (2, 130, 1000), (1, 1024, 768), (1, 1200, 1500)]


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("batch,rows,cols", ORTHO)
def test_orthogonalize(tt, batch, rows, cols, dtype):
    gen = torch.Generator().manual_seed(rows * 7 + cols)
    g = (torch.randn(batch, rows, cols, generator=gen) * 1e-3).to(dtype)
    out = tt.tt_orthogonalize(g.cuda())
    ref.check_ortho(out.cpu(), g, "ortho")
    assert torch.equal(tt.tt_orthogonalize(g.cuda()), out)
    # other steps, into a view of wider rows, from one
    wide = torch.zeros(batch, rows, cols + 5, dtype=dtype, device="cuda")
    wide[:, :, :cols] = g.cuda()
    steps = ((2.0, -1.5, 0.5), (1.875, -1.25, 0.375))
    tt.tt_orthogonalize(wide[:, :, :cols], steps=2, coefficients=steps, out=wide[:, :, :cols])
    ref.check_ortho(wide[:, :, :cols].cpu(), g, "ortho in place", steps=2, coefficients=steps)
    assert bool((wide[:, :, cols:] == 0).all())
    if batch == 1:
        assert torch.equal(tt.tt_orthogonalize(g[0].cuda()), out[0])


@pytest.mark.parametrize("rows,cols", [(8, 12), (64, 512), (200, 150)])
def test_orthogonalize_special_matrices(tt, rows, cols):
    gen = torch.Generator().manual_seed(5)
    base = torch.randn(rows, cols, generator=gen)
    g = torch.stack([base, torch.zeros(rows, cols), base * 1e-25, base * 1e25, base.clone(), base.clone(), base * 0])
    g[4, 2, 3], g[5, 0, 0], g[6, 1, 1] = math.nan, math.inf, 1e-3
    out = tt.tt_orthogonalize(g.cuda(), eps=0.0).cpu()
    ref.check_ortho(out[:1], g[:1], "plain", eps=0.0)
    ref.check_ortho(out[2:4], g[2:4], "small and large", eps=0.0)
    ref.check_ortho(out[6:], g[6:], "one entry", eps=0.0)
    assert bool(torch.isnan(out[4:6]).all())
    assert bool((tt.tt_orthogonalize(g.cuda())[1] == 0).all())


@pytest.mark.parametrize("sizes", [((5, 1000, 1000),), ((3, 8, 8), (1, 64, 512), (1, 700, 333))])
def test_orthogonalize_graph(tt, sizes):
    for batch, rows, cols in sizes:
        g = torch.randn(batch, rows, cols, device="cuda")
        tt.tt_orthogonalize(g)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = tt.tt_orthogonalize(g)
        for i in range(3):
            g.copy_(torch.randn(batch, rows, cols, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda"))
            want = tt.tt_orthogonalize(g).clone()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), i


def core_update64(table, cores, grads, momenta, lr, mu, nesterov):
    new, mom, allowed = [], [], []
    for k in range(3):
        r, n, d = table.r, table.n, table.d
        m = mu * momenta[k].double() + grads[k].double()
        u = grads[k].double() + mu * m if nesterov else m
        rows, cols = (d[0], r[1]) if k == 0 else (r[k], d[k] * r[k + 1])
        u = u.view(r[k], n[k], -1).permute(1, 0, 2).reshape(n[k], rows, cols)
        back = lambda o: o.reshape(n[k], r[k], -1).permute(1, 0, 2).reshape(-1)
        o = ref.ortho(u)
        off = (ref.ortho(u.float(), dtype=torch.float32).double() - o).norm()
        rate = lr * max(1.0, rows / cols) ** 0.5
        new.append(cores[k].double() - rate * back(o))
        mom.append(m)
        allowed.append(rate * (3 * off + 16 * ref.U * o.norm()) + 2 * ref.U * new[k].norm())
    return new, mom, allowed


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("n,d,R", [((10, 10, 10), (2, 2, 4), (4, 4)), ((61, 67, 63), (2, 4, 6), (12, 20)), ((20, 25, 20), (4, 8, 4), (32, 32)),
                                   ((9, 40, 11), (4, 8, 4), (64, 64)), ((3, 4, 5), (2, 4, 2), (128, 128)), ((1, 1, 1), (1, 1, 1), (1, 1))])
def test_core_update(tt, n, d, R, nesterov):
    r = (1, R[0], R[1], 1)
    gen = torch.Generator().manual_seed(1)
    mk = lambda std: [torch.randn(r[k] * n[k] * d[k] * r[k + 1], generator=gen) * std for k in range(3)]
    cores, grads, momenta = mk(0.05), mk(1e-3), mk(1e-2)
    if n[1] > 1:
        for t in (grads, momenta):
            t[1].view(r[1], n[1], -1)[:, 1] = 0
    table = tt.Table(n[0] * n[1] * n[2], n, d, r, [c.cuda() for c in cores])
    mom = [m.cuda() for m in momenta]
    tt.tt_core_ortho_update(table, [g.cuda() for g in grads], mom, 0.02, momentum=0.9, nesterov=nesterov)
    new, want_mom, allowed = core_update64(table, cores, grads, momenta, 0.02, 0.9, nesterov)
    for k in range(3):
        err = float((table.cores[k].cpu().double() - new[k]).norm())
        assert err <= float(allowed[k]), (k, err, float(allowed[k]))
        ref.check(mom[k].cpu(), want_mom[k], 3 * ref.U * (want_mom[k].abs() + momenta[k].double().abs()), "momentum %d" % k)
    if n[1] > 1:
        assert torch.equal(table.cores[1].cpu().view(r[1], n[1], -1)[:, 1], cores[1].view(r[1], n[1], -1)[:, 1])
    # the same bits again
    table2 = tt.Table(n[0] * n[1] * n[2], n, d, r, [c.cuda() for c in cores])
    tt.tt_core_ortho_update(table2, [g.cuda() for g in grads], [m.cuda() for m in momenta], 0.02, momentum=0.9, nesterov=nesterov)
    assert all(torch.equal(a, b) for a, b in zip(table.cores, table2.cores))


# ---- the framework's own paths ---------------------------------------------------------------------
def _bags(gen, rows, bags, most):
    lens = torch.randint(0, most + 1, (bags,), generator=gen)
    off = torch.zeros(bags, dtype=torch.int64)
    off[1:] = lens.cumsum(0)[:-1]
    return torch.randint(0, rows, (int(lens.sum()),), generator=gen), off


def _dense_rows(n, d, r, cores):
    """All rows of a table from its three cores, in 64 bits."""
    a, b, c = (x.view(r[k], n[k], d[k], r[k + 1]) for k, x in enumerate(cores))
    ab = torch.einsum("iap,pjbq->ijabq", a[0], b)
    return torch.einsum("ijabq,qkc->ijkabc", ab, c[..., 0]).reshape(n[0] * n[1] * n[2], -1)


@pytest.mark.parametrize("fuse", [False, True])
def test_projected_collection_and_optimizer(tt, fuse):
    """Bags, their projections, a loss, gradients, one orthogonalised step: the whole of it against 64 bits."""
    torch.manual_seed(0)
    gen = torch.Generator().manual_seed(3)
    shapes = [(60, (3, 4, 5)), (200, (5, 8, 5)), (24, (2, 3, 4))]
    tables = [tt.TTEmbeddingBag(rows, 16, n, (2, 2, 4), (4, 4), projection=24, projection_activation="silu") for rows, n in shapes]
    with torch.no_grad():
        for t in tables:
            t.projection.bias.normal_(0, 0.1)
    model = tt.TTEmbeddingBagCollection(tables, fuse=fuse)
    inputs = [_bags(gen, rows, bags, 4) for (rows, _), bags in zip(shapes, (17, 1, 40))]
    opt = tt.TTOrthoSGD(model, lr=0.01, momentum=0.9, other_lr=0.05)
    assert sorted(g["kind"] for g in opt.param_groups) == ["cores", "matrices", "rest"]
    outs = model([(i.cuda(), o.cuda()) for i, o in inputs])
    weights = [torch.randn(o.shape, generator=gen) for o in outs]
    before = [[p.detach().cpu().clone() for p in t.cores()] + [t.projection.weight.detach().cpu().clone(), t.projection.bias.detach().cpu().clone()] for t in tables]
    sum((o * w.cuda()).sum() for o, w in zip(outs, weights)).backward()
    opt.step()
    if fuse:
        unit = model.fused[0]
        where = [pos for _, pos in model._where]
        part = lambda t, k: unit.member_core(where[t], k).reshape(-1)
        after = [[part(t, k).detach().cpu() for k in range(3)] + [unit.projection.weight[where[t]].detach().cpu(), unit.projection.bias[where[t]].detach().cpu()]
                 for t in range(3)]
    else:
        after = [[p.detach().cpu() for p in t.cores()] + [t.projection.weight.detach().cpu(), t.projection.bias.detach().cpu()] for t in tables]
    for t, ((rows, n), (idx, off)) in enumerate(zip(shapes, inputs)):
        leaves = [b.double().requires_grad_(True) for b in before[t]]
        table = _dense_rows(n, (2, 2, 4), (1, 4, 4, 1), leaves[:3])
        pooled = torch.nn.functional.embedding_bag(idx, table, off, mode="sum")
        out = ref.act64(pooled @ leaves[3].t() + leaves[4], "silu")
        assert float((outs[t].detach().cpu().double() - out.detach()).abs().max()) <= 1e-5 * float(out.detach().abs().max()) + 1e-6
        grads = torch.autograd.grad((out * weights[t].double()).sum(), leaves)
        r, d = (1, 4, 4, 1), (2, 2, 4)
        for k in range(5):
            u = 1.9 * grads[k]  # the first step: g + 0.9 g
            if k < 3:
                shape = (d[0], r[1]) if k == 0 else (r[k], d[k] * r[k + 1])
                o = ref.ortho(u.view(r[k], n[k], -1).permute(1, 0, 2).reshape(n[k], *shape))
                o = max(1.0, shape[0] / shape[1]) ** 0.5 * o.reshape(n[k], r[k], -1).permute(1, 0, 2).reshape(-1)
            elif k == 3:
                o = 24 ** 0.5 / 16 ** 0.5 * ref.ortho(u[None])[0]
            else:
                o = u
            want = before[t][k].double() - (0.05 if k == 4 else 0.01) * o
            # steps of size 0.01; small singular values take errors of the gradients (1e-6 of the largest) up 485 times
            tol = 5e-4 * 0.01 if k < 4 else 1e-5 * float(o.abs().max()) * 0.05
            step = (after[t][k].double() - want).abs().max() if k != 0 else (after[t][k].double().reshape(want.shape) - want).abs().max()
            assert float(step) <= tol + 4 * ref.U, (t, k, float(step))


def test_projection_of_one_table_and_its_bf16_forward(tt):
    gen = torch.Generator().manual_seed(4)
    bag = tt.TTEmbeddingBag(4000, 128, (16, 16, 16), (4, 8, 4), (32, 32), projection=48, projection_activation="gelu")
    idx, off = _bags(gen, 4000, 33, 5)
    out = bag(idx.cuda(), off.cuda())
    assert out.shape == (33, 48)
    plain = tt.TTEmbeddingBag(4000, 128, (16, 16, 16), (4, 8, 4), (32, 32))
    with torch.no_grad():
        for a, b in zip(plain.cores(), bag.cores()):
            a.copy_(b)
        assert torch.equal(bag.projection(plain(idx.cuda(), off.cuda())), out)
        assert torch.equal(bag.projection(plain.forward_bf16(idx.cuda(), off.cuda())), bag.forward_bf16(idx.cuda(), off.cuda()))
    assert set(plain.state_dict()) == {"core0", "core1", "core2"}


def test_dense_module(tt):
    gen = torch.Generator(device="cuda").manual_seed(0)
    layer = tt.TTDense(40, 24, activation="relu", groups=3, dtype=torch.bfloat16, generator=gen)
    x = torch.randn(50, 40, device="cuda").bfloat16()
    off = torch.tensor([0, 20, 20, 50], device="cuda")
    assert torch.equal(layer(x, off), tt.tt_dense_forward(x, layer.weight, layer.bias, None, "relu", offsets=off))
    with pytest.raises(ValueError):
        layer(x)
    with pytest.raises(ValueError):
        tt.TTDense(4, 4, activation="tanh")
    with pytest.raises(ValueError):
        tt.TTDense(4, 4, dtype=torch.float64)
    assert tt.TTDense(4, 4, bias=False).bias is None


def test_no_graph_is_built_without_gradients(tt):
    x, w, bias, res, _ = make(9, 16, 8, torch.float32)
    assert not tt.tt_dense(x, w, bias, res, "gelu").requires_grad
    w.requires_grad_(True)
    with torch.no_grad():
        assert not tt.tt_dense(x, w, bias, res, "gelu").requires_grad
    assert tt.tt_dense(x, w, bias, res, "gelu").requires_grad


def test_optimizer_state_keeps_its_precision(tt):
    layer = tt.TTDense(24, 16, dtype=torch.bfloat16)
    opt = tt.TTOrthoSGD(layer, lr=0.01)
    for i in range(3):
        layer(torch.randn(40, 24, device="cuda").bfloat16()).float().square().mean().backward()
        opt.step()
    other = tt.TTDense(24, 16, dtype=torch.bfloat16)
    again = tt.TTOrthoSGD(other, lr=0.5)
    again.load_state_dict(opt.state_dict())
    for a, b in ((layer.weight, other.weight), (layer.bias, other.bias)):
        m = again.state[b]["momentum"]
        assert m.dtype == torch.float32 and torch.equal(m, opt.state[a]["momentum"]) and m.data_ptr() != opt.state[a]["momentum"].data_ptr()
    assert again.param_groups[0]["lr"] == 0.01


def test_many_small_matrices(tt):
    g = torch.randn(70000, 4, 6, generator=torch.Generator().manual_seed(1)) * 1e-2
    out = tt.tt_orthogonalize(g.cuda()).cpu()
    ref.check_ortho(out[::5000], g[::5000], "many")
    ref.check_ortho(out[-3:], g[-3:], "many, the last")


def test_rows_past_32_bits(tt):
    """Rows whose elements lie beyond 2^31: the last rows of a tall operand, forward and backward."""
    rows, k, n = (1 << 31) // 72 + 1000, 72, 8
    x = torch.zeros(rows, k, dtype=torch.bfloat16, device="cuda")
    x[-5:] = torch.randn(5, k, device="cuda").bfloat16()
    w = torch.randn(n, k, device="cuda").bfloat16()
    out = tt.tt_dense_forward(x, w)
    want, tol, _, _ = ref.forward64(x[-5:].cpu(), w.cpu())
    ref.check(out[-5:].cpu(), want, tol, "the last rows")
    assert float(out[:-5].abs().max()) == 0
    grad = torch.zeros(rows, n, dtype=torch.bfloat16, device="cuda")
    grad[-5:] = torch.randn(5, n, device="cuda").bfloat16()
    dx, dw, db = tt.tt_dense_backward(x, w, grad)
    (wx, ww, wb), (tx, tw, tb) = ref.backward64(x[-5:].cpu(), w.cpu(), grad[-5:].cpu())
    ref.check(dx[-5:].cpu(), wx, tx, "dx")
    ref.check(dw.cpu(), ww, tw, "dw")
    ref.check(db.cpu(), wb, tb, "dbias")
    off = torch.tensor([0, rows - 3, rows], device="cuda")
    g2 = tt.tt_dense_forward(x, torch.stack([w, -w]), offsets=off)
    assert torch.equal(g2[-5:-3], out[-5:-3]) and torch.equal(g2[-3:], -out[-3:])


def test_autograd_in_a_graph(tt):
    """A training pass through autograd, captured and replayed over new inputs with eager passes between."""
    x, w, bias, res, grad = make(500, 64, 96, torch.bfloat16, 2)
    off = torch.tensor([0, 200, 500], device="cuda")
    leaves = [t.detach().clone().requires_grad_(True) for t in (x, w, bias, res)]

    def step():
        out = tt.tt_dense(*leaves, "gelu", offsets=off)
        return (out.detach(),) + torch.autograd.grad(out, leaves, grad)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(3):
        with torch.no_grad():
            leaves[0].copy_(torch.randn(500, 64, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda"))
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), i


def test_update_in_a_graph(tt):
    n, d, r = (5, 40, 6), (4, 8, 4), (1, 64, 64, 1)
    gen = torch.Generator(device="cuda").manual_seed(0)
    mk = lambda std: [torch.randn(r[k] * n[k] * d[k] * r[k + 1], generator=gen, device="cuda") * std for k in range(3)]
    cores, grads, momenta = mk(0.05), mk(1e-3), mk(1e-2)
    copies = [[t.clone() for t in ts] for ts in (cores, momenta)]
    table, other = tt.Table(n[0] * n[1] * n[2], n, d, r, cores), tt.Table(n[0] * n[1] * n[2], n, d, r, copies[0])
    tt.tt_core_ortho_update(table, grads, momenta, 0.0, momentum=1.0, nesterov=False)  # (before the capture)
    for t, c in zip(momenta, copies[1]):
        t.copy_(c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tt.tt_core_ortho_update(table, grads, momenta, 0.01)
    for i in range(3):
        for g in grads:
            g.mul_(-0.7)
        tt.tt_core_ortho_update(other, grads, copies[1], 0.01)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(table.cores + momenta, other.cores + copies[1])), i


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_thin_sides(tt, dtype):
    """One column in or out, one row of very many columns."""
    for rows, k, n in ((3000, 1, 5), (3000, 5, 1), (1, 1, 70000), (1, 70000, 1), (70, 3, 300), (2000, 300, 3)):
        x, w, bias, res, grad = make(rows, k, n, dtype)
        want, tol, z, _ = ref.forward64(*cpu(x, w, bias, res), "silu")
        ref.check(tt.tt_dense_forward(x, w, bias, res, "silu").cpu(), want, tol, "out")
        pre = z.to(dtype)
        wants, tols = ref.backward64(*cpu(x, w, grad), pre, "silu")
        for got, want, tol, name in zip(tt.tt_dense_backward(x, w, grad, pre.cuda(), "silu"), wants, tols, ("dx", "dw", "dbias")):
            ref.check(got.cpu(), want, tol, (name, rows, k, n))
