"""`torch.nn.EmbeddingBag`-style module over the TT embedding-bag library (sum pooling).

The paper presents its operator as a drop-in replacement for PyTorch's EmbeddingBag whose
trainable parameters are the TT cores (Sections III-A and IV, "compatible with PyTorch").  This
module only wires the C-ABI calls into autograd: the index reorder of the batch is built once in
forward and reused by backward (Sections III-C / III-E), every arithmetic step runs in the HIP
kernels, and there is no CPU fallback.

Two ways to train:
  * default: backward returns core-shaped gradients for the three parameters, so any
    torch.optim optimizer can be used;
  * `fused_sgd_lr=lr`: backward applies `G <- G - lr * dG` inside the backward kernels
    (Section III-F, fused TT-core update) and reports no gradient for the cores.

Two more forward routes of the library are selectable:
  * `forward_route="sample"`: sample-level reuse (Section III-B reuse equation) on top of the reuse
    buffer of prefix products -- same bag sums, one chain per (bag, prefix) group; backward is
    unchanged (it only needs the plan);
  * `bf16_inference()` / `forward_bf16(...)`: forward on bf16 copies of the cores with fp32
    accumulation, for inference (no gradient); the copies are refreshed on request.

`projection=width` puts a dense layer of the table's own behind the pooled rows (mixed-dimension tables): `TTDense`, the
product with bias, activation and residual in one kernel, and in a fused module the product grouped by table.  `tt_dense` is
the differentiable call, `TTOrthoSGD` the optimizer whose updates of cores and dense weights are orthogonalised.

`TTFusedEmbeddingBags` holds SEVERAL tables of equal column factors and ranks as one fused TT table
(cores side by side along the row-factor axis) and serves all of them with one reorder, one forward
and one backward: what a model with many small tables needs to fill the GPU.
"""
from __future__ import annotations

import math

import torch

from . import binding


class _TTBagFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, core0, core1, core2, indices, offsets, module):
        table = module._table((core0, core1, core2))
        plan = binding.tt_index_reorder(table, indices, offsets)
        if module.forward_route == "sample":
            out = binding.tt_emb_bag_forward_sample(table, plan, offsets)
        else:
            out = binding.tt_emb_bag_forward(table, plan, indices, offsets)
        ctx.module, ctx.table, ctx.plan = module, table, plan
        ctx.save_for_backward(indices, offsets)
        return out

    @staticmethod
    def backward(ctx, grad_out):
        indices, offsets = ctx.saved_tensors
        grad_out = grad_out.contiguous()
        if grad_out.dtype != torch.float32:
            raise TypeError("the TT embedding bag computes in float32")
        module = ctx.module
        if module.fused_sgd_lr is not None:
            binding.tt_emb_bag_backward_sgd(ctx.table, ctx.plan, indices, offsets, grad_out, module.fused_sgd_lr)
            return None, None, None, None, None, None
        dcores = binding.tt_emb_bag_backward(ctx.table, ctx.plan, indices, offsets, grad_out)
        return dcores[0], dcores[1], dcores[2], None, None, None


def _csr_offsets(input, offsets, include_last_offset):
    """torch.nn.EmbeddingBag's (input, offsets) conventions -> flat indices + CSR offsets (bags + 1)."""
    if input.dim() == 2:
        if offsets is not None:
            raise ValueError("offsets must be None for 2-D input")
        bags, length = input.shape
        offsets = torch.arange(0, (bags + 1) * length, length, dtype=torch.int64, device=input.device)
        return input.reshape(-1).contiguous(), offsets
    if input.dim() != 1 or offsets is None:
        raise ValueError("1-D input needs offsets")
    offsets = offsets.to(torch.int64)
    if not include_last_offset:  # the library takes CSR offsets of length bags + 1
        offsets = torch.cat([offsets, torch.full((1,), input.numel(), dtype=torch.int64, device=input.device)])
    return input.contiguous(), offsets.contiguous()


class _DenseFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, residual, activation, offsets):
        need = any(ctx.needs_input_grad[:3])
        pre = torch.empty((x.shape[0], w.shape[-2]), dtype=x.dtype, device=x.device) if need and activation != "none" else None
        out = binding.tt_dense_forward(x, w, bias, residual, activation, offsets=offsets, pre=pre)
        ctx.activation, ctx.has_bias, ctx.has_residual = activation, bias is not None, residual is not None
        ctx.save_for_backward(x, w, pre, offsets)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_out):
        x, w, pre, offsets = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx = dw = db = None
        if any(need[:3]):
            g = grad_out
            if g.dim() != 2 or g.stride(1) != 1 or (g.shape[0] > 1 and g.stride(0) < g.shape[1]):
                g = g.contiguous()  # an expanded gradient (of a sum) has steps of zero
            dx, dw, db = binding.tt_dense_backward(x, w, g, pre, ctx.activation, offsets=offsets,
                                                   needs=(need[0], need[1], need[2] and ctx.has_bias))
        dres = grad_out if ctx.has_residual and need[3] else None
        return dx, dw, db, dres, None, None


def _row_major(t):
    """t as the library takes it: columns next to each other, rows that do not overlap (a copy where they are not)."""
    if t is None or t.dim() != 2 or ((t.shape[1] <= 1 or t.stride(1) == 1) and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1])):
        return t
    return t.contiguous()


def tt_dense(x, w, bias=None, residual=None, activation="none", offsets=None):
    """`act(x w^T + bias) + residual`, differentiable in its four tensors; grouped by `offsets` as in
    `binding.tt_dense_forward`.  Rows of no group give zeros and get none: their residual is not added, and its gradient there
    is left out too.  With an activation in training the pre-activation is kept in x's type for the backward pass.  (As with any autograd
    function: a backward pass that is captured into a graph should accumulate into no leaf that an eager graph still holds;
    `torch.autograd.grad` does not.  There is no forward-mode derivative: tensors with tangents are refused.)"""
    train = torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, w, bias, residual))
    # inside a level of forward-mode differentiation the autograd function is asked, which refuses tensors with tangents
    dual = torch.autograd.forward_ad._current_level >= 0
    if train and residual is not None and offsets is not None and residual.requires_grad:
        residual = _GroupRows.apply(residual, offsets)
    if bias is not None and not bias.is_contiguous():
        bias = bias.contiguous()
    x, w, residual = _row_major(x), w if w.is_contiguous() else w.contiguous(), _row_major(residual)
    if not train and not dual:  # nothing is kept for a backward pass
        return binding.tt_dense_forward(x, w, bias, residual, activation, offsets=offsets)
    return _DenseFunction.apply(x, w, bias, residual, activation, offsets)


class _GroupRows(torch.autograd.Function):
    """The identity, whose gradient is zero in rows of no group."""

    @staticmethod
    def forward(ctx, t, offsets):
        ctx.save_for_backward(offsets)
        return t.view_as(t)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        (offsets,) = ctx.saved_tensors
        row = torch.arange(grad.shape[0], device=grad.device)
        return torch.where(((row >= offsets[0]) & (row < offsets.max()))[:, None], grad, torch.zeros((), dtype=grad.dtype, device=grad.device)), None


class TTDense(torch.nn.Module):
    """Dense layer `act(x weight^T + bias) + residual` in one kernel: weight [out, in], or with `groups` [groups, out, in] where
    group g's serves the rows offsets[g] .. offsets[g + 1] of x (offsets int64 [groups + 1] on the device).
    activation: "none", "relu", "gelu", "silu" or "sigmoid"; dtype float32, bfloat16 or float16."""

    def __init__(self, in_features: int, out_features: int, bias: bool = True, activation: str = "none", groups=None, device="cuda",
                 dtype=torch.float32, generator=None):
        super().__init__()
        if activation not in binding.ACTIVATIONS:
            raise ValueError("activation is one of %s" % ", ".join(binding.ACTIVATIONS))
        if dtype not in binding.DTYPES:
            raise ValueError("dtype is float32, bfloat16 or float16")
        self.in_features, self.out_features, self.activation = int(in_features), int(out_features), activation
        self.groups = None if groups is None else int(groups)
        lead = () if groups is None else (self.groups,)
        w = torch.empty(lead + (self.out_features, self.in_features), dtype=torch.float32, device=device)
        w.normal_(0.0, self.in_features ** -0.5, generator=generator)
        self.weight = torch.nn.Parameter(w.to(dtype))
        self.bias = torch.nn.Parameter(torch.zeros(lead + (self.out_features,), dtype=dtype, device=device)) if bias else None

    def forward(self, x, offsets=None, residual=None):
        if (offsets is None) != (self.groups is None):
            raise ValueError("offsets go with groups")
        return tt_dense(x, self.weight, self.bias, residual, self.activation, offsets)

    def extra_repr(self) -> str:
        return "%d -> %d%s, %s" % (self.in_features, self.out_features, "" if self.groups is None else ", %d groups" % self.groups, self.activation)


class _Projected(torch.nn.Module):
    """A module that may have a `projection`; one that was pickled before there were any has none."""

    def __setstate__(self, state):
        super().__setstate__(state)
        if "projection" not in self.__dict__ and "projection" not in self._modules:
            self.projection = None


class TTEmbeddingBag(_Projected):
    """Sum-pooling embedding bag whose table of `num_embeddings x embedding_dim` is held as three
    TT cores `G_k[r_k][n_k][d_k][r_{k+1}]` (flat float32 parameters `core0..core2`).

    n, d     row / column factors: prod(n) >= num_embeddings, prod(d) == embedding_dim
    ranks    (R1, R2)
    forward(input, offsets=None) follows torch.nn.EmbeddingBag: 1-D `input` with `offsets`
    (bag starts; with include_last_offset the last entry is len(input)), or 2-D `input` whose rows
    are bags of equal length.  Not supported (raise): per_sample_weights, padding_idx, max_norm,
    modes other than "sum".
    projection  width of a dense layer of the table's own behind the pooled rows (None: there is none), with
    projection_activation (`TTDense`); the outputs are then [bags x projection]
    """

    def __init__(self, num_embeddings: int, embedding_dim: int, n, d, ranks, mode: str = "sum",
                 include_last_offset: bool = False, init_row_std: float = 0.1, fused_sgd_lr=None,
                 forward_route: str = "batch", device="cuda", generator=None, projection=None,
                 projection_activation: str = "none"):
        super().__init__()
        if mode != "sum":
            raise NotImplementedError("only sum pooling is defined for the TT embedding bag")
        n, d, ranks = tuple(int(x) for x in n), tuple(int(x) for x in d), tuple(int(x) for x in ranks)
        if len(n) != 3 or len(d) != 3 or len(ranks) != 2:
            raise ValueError("three row factors, three column factors and two ranks are required")
        if d[0] * d[1] * d[2] != embedding_dim:
            raise ValueError("prod(d) must equal embedding_dim")
        if n[0] * n[1] * n[2] < num_embeddings:
            raise ValueError("prod(n) must be at least num_embeddings")
        self.num_embeddings, self.embedding_dim = int(num_embeddings), int(embedding_dim)
        self.n, self.d, self.r = n, d, (1, ranks[0], ranks[1], 1)
        self.include_last_offset = bool(include_last_offset)
        self.fused_sgd_lr = None if fused_sgd_lr is None else float(fused_sgd_lr)
        if forward_route not in ("batch", "sample"):
            raise ValueError("forward_route is 'batch' (each distinct row once, then a bag sum) or 'sample'")
        self.forward_route = forward_route
        self._bf16_cores = None
        # a row entry is a sum of R1*R2 products of three core entries: choose the core scale so that
        # the rows start with standard deviation `init_row_std`
        s = (init_row_std ** 2 / (ranks[0] * ranks[1])) ** (1.0 / 6.0)
        for k in range(3):
            numel = self.r[k] * n[k] * d[k] * self.r[k + 1]
            w = torch.empty(numel, dtype=torch.float32, device=device)
            w.normal_(0.0, s, generator=generator)
            self.register_parameter("core%d" % k, torch.nn.Parameter(w))
        self.projection = None if projection is None else TTDense(embedding_dim, projection, activation=projection_activation, device=device,
                                                                  generator=generator)

    def cores(self):
        return [self.core0, self.core1, self.core2]

    def _table(self, cores) -> binding.Table:
        return binding.Table(self.num_embeddings, self.n, self.d, self.r, [c.detach() for c in cores])

    def _bag_offsets(self, input, offsets):
        return _csr_offsets(input, offsets, self.include_last_offset)

    def forward(self, input, offsets=None, per_sample_weights=None):
        if per_sample_weights is not None:
            raise NotImplementedError("per_sample_weights are not defined for the TT embedding bag")
        if not input.is_cuda or not self.core0.is_cuda:
            raise RuntimeError("the TT embedding bag runs on the GPU only (there is no CPU path)")
        if input.dtype != torch.int64:
            input = input.to(torch.int64)
        indices, offsets = self._bag_offsets(input, offsets)
        out = _TTBagFunction.apply(self.core0, self.core1, self.core2, indices, offsets, self)
        return out if self.projection is None else self.projection(out)

    def bf16_inference(self):
        """(Re)build the bf16 copies of the cores that `forward_bf16` reads; call again after the cores
        have changed.  Only for shapes the matrix-core kernels serve (the library refuses others)."""
        self._bf16_cores = binding.tt_cores_to_bf16(self._table(self.cores()))
        return self

    @torch.no_grad()
    def forward_bf16(self, input, offsets=None):
        """Inference forward on the bf16 copies of the cores (fp32 accumulation); no autograd graph.
        Short batches are summed without a plan, in another order: a bag's last bits follow the sizes of its batch."""
        if self._bf16_cores is None:
            self.bf16_inference()
        if input.dtype != torch.int64:
            input = input.to(torch.int64)
        indices, offsets = self._bag_offsets(input, offsets)
        table = self._table(self.cores())
        # the plan would serve this call only: short batches are faster without one
        if binding.tt_forward_bf16_direct_pays(table, indices.numel(), offsets.numel() - 1):
            out = binding.tt_emb_bag_forward_bf16_direct(table, self._bf16_cores, indices, offsets)
        else:
            plan = binding.tt_index_reorder(table, indices, offsets)
            out = binding.tt_emb_bag_forward_bf16(table, self._bf16_cores, plan, offsets)
        return out if self.projection is None else self.projection(out)

    def extra_repr(self) -> str:
        return "%d x %d, n=%s, d=%s, ranks=%s, %.1fx smaller than dense%s" % (
            self.num_embeddings, self.embedding_dim, self.n, self.d, self.r[1:3],
            self.num_embeddings * self.embedding_dim / float(sum(c.numel() for c in self.cores())),
            ", fused SGD lr=%g" % self.fused_sgd_lr if self.fused_sgd_lr is not None else "")

    @staticmethod
    def near_cubic_factors(num_embeddings: int):
        """Three near-equal row factors whose product covers `num_embeddings`."""
        n3 = 1
        while n3 ** 3 < num_embeddings:
            n3 += 1
        n2 = 1
        while n2 * n2 * n3 < num_embeddings:
            n2 += 1
        n1 = max(1, -(-num_embeddings // (n2 * n3)))
        return (n1, n2, n3)


class TTFusedEmbeddingBags(_Projected):
    """Several sum-pooling embedding bags of one embedding_dim, one set of column factors `d` and one
    pair of ranks, held as ONE fused TT table: core k is `[r_k][sum of the tables' n_k][d_k][r_k+1]`
    and table t owns a range of the middle axis of every core.  A row of table t is the product of
    its own three slices (TT-matrix equation, Section II-B; index split per table, Section III-B), so
    outputs and gradients are those of the separate tables -- computed with one reorder, one forward
    and one backward for all of them.

    tables    list of `(num_embeddings, (n1, n2, n3))`; the sums of the row factors must keep the
              fused row count below 2^31 (split the tables over several modules otherwise:
              `binding.fusion_groups` deals them out)
    forward(inputs) takes one `(input, offsets)` pair (or a 2-D `input`) per table, as
    `TTEmbeddingBag.forward` does, and returns the list of pooled outputs in table order (views of
    one `[all bags x embedding_dim]` tensor).  `fused_sgd_lr` as for `TTEmbeddingBag`.
    projection  width of a dense layer behind the pooled rows, a weight for every table (`TTDense` grouped by
    table: one product for all), with projection_activation; outputs are then [bags x projection]
    """

    def __init__(self, tables, embedding_dim: int, d, ranks, include_last_offset: bool = False,
                 init_row_std: float = 0.1, fused_sgd_lr=None, device="cuda", generator=None, projection=None,
                 projection_activation: str = "none"):
        super().__init__()
        d, ranks = tuple(int(x) for x in d), tuple(int(x) for x in ranks)
        if len(d) != 3 or len(ranks) != 2 or d[0] * d[1] * d[2] != embedding_dim:
            raise ValueError("three column factors with prod(d) == embedding_dim and two ranks are required")
        tables = [(int(rows), tuple(int(x) for x in n)) for rows, n in tables]
        for rows, n in tables:
            if len(n) != 3 or n[0] * n[1] * n[2] < rows:
                raise ValueError("every table needs three row factors with prod(n) >= num_embeddings")
        self.tables, self.embedding_dim = tables, int(embedding_dim)
        self.d, self.r = d, (1, ranks[0], ranks[1], 1)
        self.include_last_offset = bool(include_last_offset)
        self.fused_sgd_lr = None if fused_sgd_lr is None else float(fused_sgd_lr)
        self.forward_route = "batch"
        self.n = tuple(sum(n[k] for _, n in tables) for k in range(3))
        self.num_embeddings = self.n[0] * self.n[1] * self.n[2]  # rows of the fused table
        if self.num_embeddings >= 2 ** 31 - 1:
            raise ValueError("the fused table would have 2^31 rows or more: fuse fewer tables")
        self._fused = None  # binding.FusedLayout, built on first use (it needs the library)
        s = (init_row_std ** 2 / (ranks[0] * ranks[1])) ** (1.0 / 6.0)
        for k in range(3):
            w = torch.empty(self.r[k] * self.n[k] * d[k] * self.r[k + 1], dtype=torch.float32, device=device)
            w.normal_(0.0, s, generator=generator)
            self.register_parameter("core%d" % k, torch.nn.Parameter(w))
        self.projection = None if projection is None else TTDense(embedding_dim, projection, activation=projection_activation,
                                                                  groups=len(tables), device=device, generator=generator)

    def cores(self):
        return [self.core0, self.core1, self.core2]

    def member_core(self, t: int, k: int, core=None):
        """Table t's part of fused core k (or of a tensor of its size, e.g. `.grad`): a strided view
        `[r_k][n_k(t)][d_k][r_k+1]`."""
        core = self.cores()[k] if core is None else core
        o = sum(n[k] for _, n in self.tables[:t])
        return core.view(self.r[k], self.n[k], self.d[k], self.r[k + 1])[:, o:o + self.tables[t][1][k]]

    def _table(self, cores) -> binding.Table:
        return binding.Table(self.num_embeddings, self.n, self.d, self.r, [c.detach() for c in cores])

    def forward(self, inputs):
        inputs = list(inputs)
        if len(inputs) != len(self.tables):
            raise ValueError("one input per table: got %d for %d tables" % (len(inputs), len(self.tables)))
        if not self.core0.is_cuda:
            raise RuntimeError("the TT embedding bag runs on the GPU only (there is no CPU path)")
        idx, off = [], []
        for x in inputs:
            inp, o = x if isinstance(x, (tuple, list)) else (x, None)
            if inp.dtype != torch.int64:
                inp = inp.to(torch.int64)
            i, o = self._bag_offsets(inp, o)
            idx.append(i)
            off.append(o)
        if self._fused is None:
            self._fused = binding.FusedLayout(self.tables)
        # (a call's own, written on the device: a captured call keeps its memory, and no other call sees it)
        ranges = None if self.projection is None else torch.empty(len(self.tables) + 1, dtype=torch.int64, device=off[0].device)
        f_idx, f_off = self._fused.fuse_lookups(idx, off, starts=not self.include_last_offset, ranges=ranges)
        out = _TTBagFunction.apply(self.core0, self.core1, self.core2, f_idx, f_off, self)
        bags = tuple(o.numel() - (1 if self.include_last_offset else 0) for o in off)
        if self.projection is not None:
            out = self.projection(out, ranges)
        return list(torch.split(out, bags))

    def _bag_offsets(self, input, offsets):
        """Flat indices and CSR offsets, or (without include_last_offset) bag starts as they are given: the
        map into the fused table knows where the last bag ends, so nothing is appended to them (26 tables:
        52 small launches and 350 us of host time a pass)."""
        if self.include_last_offset or input.dim() != 1 or offsets is None:
            input, offsets = _csr_offsets(input, offsets, self.include_last_offset)
            return input, offsets if self.include_last_offset else offsets[:-1]
        if offsets.dim() != 1 or offsets.device != input.device:
            raise ValueError("offsets must be a 1-D tensor on the device of the input")
        return input.contiguous(), offsets.to(torch.int64).contiguous()

    def extra_repr(self) -> str:
        return "%d tables fused into %s rows x %d, d=%s, ranks=%s" % (
            len(self.tables), "x".join(str(x) for x in self.n), self.embedding_dim, self.d, self.r[1:3])


class TTEmbeddingBagCollection(torch.nn.Module):
    """The sparse side of a DLRM: one `TTEmbeddingBag` per categorical feature (Section IV: the TT
    tables replace the model's embedding tables one for one).

    tables    iterable of `TTEmbeddingBag`, or of keyword dicts for its constructor
    streams   number of side streams the tables are dealt to in forward (1: the current stream).
              Tables are independent and a table's kernels are short, so several streams let the
              GPU overlap them; autograd runs a table's backward on the stream of its forward.
    fuse      store tables of one family (same column factors, ranks, offset convention and update
              mode) as fused tables (`TTFusedEmbeddingBags`, dealt out by `binding.fusion_groups`) and
              serve each fused table with one set of launches.  The parameters are then the fused
              cores (`self.fused[g].core0..2`; `member_core` gives a table's part); the given tables'
              core values are copied in.  `fuse_groups`: number of fused tables per family (None: the
              fewest the limits allow).
    forward(inputs) takes one `(input, offsets)` pair (or a 2-D `input`) per table and returns the
    list of pooled outputs `[bags x embedding_dim]`, in table order.
    """

    def __init__(self, tables, streams: int = 1, fuse: bool = False, fuse_groups=None):
        super().__init__()
        tables = [t if isinstance(t, TTEmbeddingBag) else TTEmbeddingBag(**t) for t in tables]
        if streams < 1:
            raise ValueError("streams must be at least 1")
        self.num_streams = int(streams)
        self._side = None
        self.num_tables = len(tables)
        if not fuse:
            self.tables = torch.nn.ModuleList(tables)
            self.fused, self._where = None, None
            return
        self.tables = None
        families = {}
        for t, bag in enumerate(tables):
            p = bag.projection
            key = (bag.d, bag.r, bag.include_last_offset, bag.fused_sgd_lr, bag.core0.device, p and (p.out_features, p.activation))
            families.setdefault(key, []).append(t)
        fused, where = [], [None] * len(tables)
        for (d, r, last, lr, dev, proj), idxs in families.items():
            members = [(tables[t].num_embeddings, tables[t].n) for t in idxs]
            for part in binding.fusion_groups(members, groups=fuse_groups):
                m = TTFusedEmbeddingBags([members[p] for p in part], d[0] * d[1] * d[2], d, r[1:3],
                                         include_last_offset=last, fused_sgd_lr=lr, device=dev,
                                         projection=proj and proj[0], projection_activation=proj[1] if proj else "none")
                with torch.no_grad():
                    for pos, p in enumerate(part):
                        src = tables[idxs[p]]
                        for k in range(3):
                            m.member_core(pos, k).copy_(src.cores()[k].view(r[k], src.n[k], d[k], r[k + 1]))
                        if proj:
                            m.projection.weight[pos].copy_(src.projection.weight)
                            m.projection.bias[pos].copy_(src.projection.bias)
                        where[idxs[p]] = (len(fused), pos)
                fused.append(m)
        self.fused = torch.nn.ModuleList(fused)
        self._where = where

    def forward(self, inputs):
        inputs = list(inputs)
        if len(inputs) != self.num_tables:
            raise ValueError("one input per table: got %d for %d tables" % (len(inputs), self.num_tables))
        if self.fused is not None:
            per_group = [[None] * len(m.tables) for m in self.fused]
            for t, x in enumerate(inputs):
                gi, pos = self._where[t]
                per_group[gi][pos] = x
            units = [(m, xs) for m, xs in zip(self.fused, per_group)]
            run = lambda unit: unit[0](unit[1])
        else:
            pairs = [x if isinstance(x, (tuple, list)) else (x, None) for x in inputs]
            units = list(zip(self.tables, pairs))
            run = lambda unit: unit[0](unit[1][0], unit[1][1])
        if self.num_streams == 1:
            results = [run(u) for u in units]
        else:
            if self._side is None:
                self._side = [torch.cuda.Stream() for _ in range(self.num_streams)]
            cur = torch.cuda.current_stream()
            for s in self._side:
                s.wait_stream(cur)
            results = []
            for i, u in enumerate(units):
                with torch.cuda.stream(self._side[i % self.num_streams]):
                    results.append(run(u))
            for s in self._side:
                cur.wait_stream(s)
            for r in results:
                for o in (r if isinstance(r, list) else [r]):
                    o.record_stream(cur)
        if self.fused is None:
            return results
        return [results[gi][pos] for gi, pos in self._where]


class TTOrthoSGD(torch.optim.Optimizer):
    """Gradient descent whose updates are orthogonalised (`binding.tt_orthogonalize`): momentum, then
    `W <- W - lr sqrt(max(1, rows / cols)) ortho(u)` for every dense weight of the model's `TTDense` layers (every group's own)
    and for every slice of the cores of its TT bags (`binding.tt_core_ortho_update`).  Whatever else the model has (biases,
    other layers) takes plain steps of `other_lr` with the same momentum.  Momenta are float32, and so are the updates up to the
    step itself, which is rounded to the parameter's type once.

    model   a module; its parameters are sorted by the layers that own them
    Cores and weights without gradients (frozen, unused in this step, or of tables with `fused_sgd_lr`) stay as they are.
    """

    def __init__(self, model, lr: float, momentum: float = 0.95, nesterov: bool = True, steps: int = 5,
                 coefficients=binding.ORTHO_COEFFICIENTS, eps: float = 1e-7, other_lr=None):
        if lr < 0 or not 0 <= momentum < 1:
            raise ValueError("lr must not be negative, momentum is in [0, 1)")
        self._tables = [m for m in model.modules() if isinstance(m, (TTEmbeddingBag, TTFusedEmbeddingBags))]
        once = lambda ps: list({id(p): p for p in ps}.values())  # layers may share a parameter
        matrices = once(m.weight for m in model.modules() if isinstance(m, TTDense))
        cores = once(c for t in self._tables for c in t.cores())
        taken = {id(p) for p in matrices + cores}
        rest = [p for p in model.parameters() if id(p) not in taken]
        groups = [dict(params=ps, kind=kind, lr=rate) for ps, kind, rate in
                  ((cores, "cores", lr), (matrices, "matrices", lr), (rest, "rest", lr if other_lr is None else other_lr)) if ps]
        super().__init__(groups, dict(kind="rest", momentum=momentum, nesterov=nesterov, steps=steps, coefficients=coefficients, eps=eps))

    def load_state_dict(self, state_dict):
        super().load_state_dict(state_dict)  # casts what it loads to the parameters' types
        for mine, saved in zip(self.param_groups, state_dict["param_groups"]):
            for p, name in zip(mine["params"], saved["params"]):
                if name in state_dict["state"]:
                    m = state_dict["state"][name]["momentum"]
                    self.state[p]["momentum"] = m.to(device=p.device, dtype=torch.float32, copy=True).contiguous()

    def __getstate__(self):  # copies and pickles have the tables too
        return dict(super().__getstate__(), _tables=self._tables)

    def _momentum(self, p):
        state = self.state[p]
        if "momentum" not in state:
            state["momentum"] = torch.zeros_like(p, dtype=torch.float32, memory_format=torch.contiguous_format)
        return state["momentum"]

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for group in self.param_groups:
            lr, mu, how = group["lr"], group["momentum"], dict(steps=group["steps"], coefficients=group["coefficients"], eps=group["eps"])
            if group["kind"] == "cores":
                done = set()
                for t in self._tables:
                    cores = t.cores()
                    steps = [c.grad is not None and id(c) not in done for c in cores]
                    if not any(steps):
                        continue
                    done.update(id(c) for c in cores)
                    # cores are updated each by itself: one without a gradient (a frozen one), or that another table has too, has a copy stand
                    # in for it
                    binding.tt_core_ortho_update(t._table([c if s else c.clone() for c, s in zip(cores, steps)]),
                                                 [c.grad.contiguous() if s else torch.zeros_like(c) for c, s in zip(cores, steps)],
                                                 [self._momentum(c) if s else torch.zeros_like(c) for c, s in zip(cores, steps)], lr,
                                                 momentum=mu, nesterov=group["nesterov"], **how)
                continue
            for p in group["params"]:
                if p.grad is None:
                    continue
                g, buf = p.grad.float(), self._momentum(p)
                buf.mul_(mu).add_(g)
                u = torch.add(g, buf, alpha=mu) if group["nesterov"] else buf
                if group["kind"] == "matrices":
                    rows, cols = p.shape[-2:]
                    # (in float32: rounded to 16 bits first, a sum of gradients leaves float16's range, and bfloat16's 8 bits are what the
                    # steps take up to 485 times)
                    p.add_(binding.tt_orthogonalize(u.contiguous(), **how), alpha=-lr * math.sqrt(max(1.0, rows / cols)))
                else:
                    p.add_(u, alpha=-lr)
        return loss
