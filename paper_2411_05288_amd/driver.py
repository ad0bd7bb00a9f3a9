"""Host driver: runs the p shards of one configuration on one GPU, all of them in one call per pass where it can.

This is launch ordering and buffer ownership only.  It follows Algorithm 1 of the paper:
pass S on all shards (vp_output_fwd_group), barrier C1 (vp_combine_stats, standing in for the two
all-reduces), pass T on all shards (vp_output_bwd_group) with the reduce C2 realised as fp32
accumulation into one dH buffer in ascending order of the vocabulary.  With algorithm=2 it follows
Algorithm 2: pass S also forms A and B (vp_output_fwd_alg2_group), the input gradient is accumulated inside the single
barrier (vp_output_dx_alg2_gather), and pass T is dW alone.  The calls of a single
shard (vp_output_fwd, vp_output_bwd) serve plans whose shards without real rows are not the last ones, and plans
without the workspace for all shards.  All device buffers are allocated once, when the plan is built; a step
allocates nothing.
"""
from __future__ import annotations

import contextlib
from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

from . import binding as B


def _on(stream):
    """Context in which torch's own work runs on the same stream as the library's kernels."""
    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream))
    return torch.cuda.stream(stream)


@dataclass
class OutputLayerResult:
    loss: torch.Tensor            # [1] fp32
    loss_rows: torch.Tensor       # [N] fp32
    global_max: torch.Tensor      # [N]
    global_sumexp: torch.Tensor   # [N]
    local_max: torch.Tensor       # [p, N]
    local_sumexp: torch.Tensor    # [p, N]
    local_target: torch.Tensor    # [p, N]
    dH: torch.Tensor              # [N, h] fp32
    dW: List[torch.Tensor]        # p x [Vs, h] fp32
    logits: Optional[List[torch.Tensor]]


class BlockNormPlan:
    """Buffers and calls of the norms around a block: r = x + scale * gate * norm(y), H = norm(r) (``post`` norms y, ``center``
    makes layer norms of RMS norms; y=None: H = norm(x) alone), and the gradients of all of it.

    ``train=False`` keeps no statistics and no buffers for gradients: ``forward`` alone, as for single tokens.  Gradients of
    activations (dx, dy) are of ``grad_dtype`` (default: the type of x), those of parameters fp32.  A plan's calls share its
    buffers: they belong on one stream, or one after the other."""

    def __init__(self, x: torch.Tensor, y: Optional[torch.Tensor] = None, *, gate=None, w=None, b=None, w_post=None, b_post=None,
                 scale: float = 1.0, eps: float = 1e-5, post: bool = False, center: bool = False, grad_dtype=None,
                 train: bool = True):
        self.x, self.y = x, y
        self.N, self.h = x.shape
        self.gate, self.w, self.b, self.w_post, self.b_post = gate, w, b, w_post, b_post
        self.scale, self.eps, self.post, self.center = scale, eps, post, center
        f32 = dict(dtype=torch.float32, device=x.device)
        self.r = torch.empty_like(x) if y is not None else None
        self.H = torch.empty_like(x)
        self.stats = self.dx = self.dy = self.dgate = self.dw = self.db = self.dw_post = self.db_post = self.workspace = None
        if not train:
            return
        self.stats = torch.empty((4, self.N), **f32)
        self.dx = torch.empty((self.N, self.h), dtype=grad_dtype or x.dtype, device=x.device)
        self.dy = torch.empty_like(self.dx) if y is not None else None
        self.dgate, self.dw, self.db, self.dw_post, self.db_post = (
            None if t is None else torch.empty(t.shape, **f32) for t in (gate, w, b, w_post, b_post))
        self.workspace = torch.empty((B.vp_block_norm_bwd_workspace_bytes(
            self.N, self.h, 0 if gate is None else gate.shape[0], post),), dtype=torch.uint8, device=x.device)

    def forward(self, stream=None) -> None:
        B.vp_block_norm_fwd(self.x, self.y, self.H, r=self.r, stats=self.stats, gate=self.gate, w=self.w, b=self.b,
                            w_post=self.w_post, b_post=self.b_post, scale=self.scale, eps=self.eps, post=self.post,
                            center=self.center, stream=stream)

    def backward(self, dH: torch.Tensor, dr: Optional[torch.Tensor] = None, stream=None) -> None:
        if self.stats is None:
            raise B.VPError("a plan with train=False has no backward pass")
        B.vp_block_norm_bwd(dH, self.x if self.r is None else self.r, self.y, self.stats, dx=self.dx, dy=self.dy, dr=dr,
                            gate=self.gate, w=self.w, w_post=self.w_post, b_post=self.b_post, scale=self.scale, post=self.post,
                            center=self.center, dgate=self.dgate, dw=self.dw, db=self.db, dw_post=self.dw_post,
                            db_post=self.db_post, workspace=self.workspace, stream=stream)

    def parameter_gradients(self) -> List[torch.Tensor]:
        return [t for t in (self.dgate, self.dw, self.db, self.dw_post, self.db_post) if t is not None]


class GradientClipPlan:
    """The norm of many gradients together, and clipping by it: the gradients of all layers of a step, of fp32 or bf16, in place
    or into ``outs`` (tensors of their types and shapes, views of one flat buffer among them).  The plan keeps the tensors and
    their addresses: gradients that are other tensors in the next step need a new plan (``covers``), and a tensor that moved or
    changed its size or type is refused.  A plan's calls share its workspace and ``norm`` (given, or the plan's own): they belong
    on one stream, or one after the other."""

    def __init__(self, grads: List[torch.Tensor], outs: Optional[List[torch.Tensor]] = None,
                 norm: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
        self.arguments = B.GradientArguments(grads, outs)
        dev = self.arguments.grads[0].device if self.arguments.n else torch.device("cuda", torch.cuda.current_device())
        self.norm = torch.empty((1,), dtype=torch.float32, device=dev) if norm is None else norm
        if workspace is None:
            workspace = torch.empty((B.vp_grad_workspace_bytes(self.arguments.n),), dtype=torch.uint8, device=dev)
        self.workspace = workspace

    def covers(self, grads: List[torch.Tensor]) -> bool:
        """Whether it was made for exactly these tensors, and they are where and what they were."""
        a = self.arguments
        return a.n == len(grads) and all(g is mine for g, mine in zip(grads, a.grads)) and a.unchanged()

    def compute_norm(self, stream=None) -> None:
        B.vp_grad_norm(self.arguments, self.norm, self.workspace, stream)

    def clip(self, max_norm: float, stream=None) -> None:
        B.vp_grad_clip(self.arguments, max_norm, self.norm, self.workspace, stream=stream)

    def scale(self, max_norm: float, norm: Optional[torch.Tensor] = None, stream=None) -> None:
        """Clips by ``norm`` (default: what compute_norm left, or what the caller made of it, as by a sum over devices)."""
        B.vp_grad_scale(self.arguments, max_norm, self.norm if norm is None else norm, self.workspace, stream=stream)


class OutputLayerPlan:
    """Buffers and launch order for one output-layer workload of p shards.

    Shards may have different numbers of rows (a short last shard); shard r owns the global
    vocabulary rows [offsets[r], offsets[r] + rows_r).  ``vocab_size`` states the true
    vocabulary when the table was padded to split evenly (the paper pads V to a multiple of
    2p): rows at or beyond it are padding.  Padding never reaches the kernels -- a shard is
    passed as its valid prefix, which is the same as giving the padded logits -inf -- and
    the padding rows of dW are zero.

    All shards go through one call per pass, which keeps the D matrices of all of them (at most
    4 GiB) and up to 1 GiB of partial sums in ``workspace``; one shard at a time needs the largest
    D alone.  ``workspace_limit`` (bytes) makes the plan go shard by shard where the workspace
    would be larger than that, and so does a device without room for it; with algorithm=2 pass S alone
    does so where the rest fits.

    With ``norm`` (a BlockNormPlan; H is then None) the plan begins with that norm, whose H it reads, and its backward pass
    ends with the norm's, from dH.  ``clip_gradients`` clips dW and the norm's parameter gradients, and ``others`` with them, by
    the norm of all of them together."""

    def __init__(self, H: Optional[torch.Tensor], W_shards: List[torch.Tensor], labels: torch.Tensor,
                 save_logits: bool = True, grad_scale: Optional[float] = None, vocab_size: Optional[int] = None,
                 algorithm: int = 1, workspace_limit: Optional[int] = None,
                 norm: Optional["BlockNormPlan"] = None):
        if (H is None) == (norm is None):
            raise B.VPError("either H or the norm that makes it")
        self.norm, self.clip_plan, self.clip_norm, self.clip_workspaces = norm, None, None, []
        H = norm.H if H is None else H
        if algorithm not in (1, 2):
            raise B.VPError("algorithm must be 1 (two barriers) or 2 (one barrier)")
        self.algorithm = algorithm
        self.H, self.W, self.labels = H, W_shards, labels
        self.N, self.h = H.shape
        self.p = len(W_shards)
        self.rows = [int(w.shape[0]) for w in W_shards]
        self.Vs = self.rows[0]
        for w in W_shards:
            if w.dim() != 2 or w.shape[1] != self.h:
                raise B.VPError("every shard must be [rows, h]")
        self.offsets = [0]
        for n in self.rows[:-1]:
            self.offsets.append(self.offsets[-1] + n)
        total = self.offsets[-1] + self.rows[-1]
        self.vocab_size = total if vocab_size is None else int(vocab_size)
        if not 0 < self.vocab_size <= total:
            raise B.VPError("vocab_size must be in (0, total rows]")
        # valid (non-padding) rows of every shard
        self.valid = [max(0, min(n, self.vocab_size - off)) for n, off in zip(self.rows, self.offsets)]
        self.dt = B.VP_F32 if H.dtype == torch.float32 else B.VP_BF16
        self.save_logits = save_logits
        self.grad_scale = (1.0 / self.N) if grad_scale is None else float(grad_scale)
        dev = H.device
        f32 = dict(dtype=torch.float32, device=dev)
        N, h, p = self.N, self.h, self.p
        self.local_max = torch.empty((p, N), **f32)
        self.local_sumexp = torch.empty((p, N), **f32)
        self.local_target = torch.empty((p, N), **f32)
        self.global_max = torch.empty((N,), **f32)
        self.global_sumexp = torch.empty((N,), **f32)
        self.loss_rows = torch.empty((N,), **f32)
        self.loss = torch.empty((1,), **f32)
        self.dH = torch.empty((N, h), **f32)
        self.dW = [torch.empty((n, h), **f32) for n in self.rows]
        self.logits = ([torch.empty((N, max(v, 1)), dtype=H.dtype, device=dev) for v in self.valid]
                       if save_logits else None)
        flags = B.VP_SAVE_LOGITS if save_logits else 0
        fwd_call = B.VP_CALL_OUTPUT_FWD if algorithm == 1 else B.VP_CALL_OUTPUT_FWD_ALG2
        nbytes = 256
        for v in self.valid:
            if v > 0:
                nbytes = max(nbytes, B.vp_workspace_bytes(fwd_call, N, h, v, self.dt, flags),
                             B.vp_workspace_bytes(B.VP_CALL_OUTPUT_BWD, N, h, v, self.dt, flags))
        # All shards of the device go through one call when the ones with real rows come first (else one by one); that
        # call's workspace is larger: the D matrices of all shards (at most 4 GiB) and the slices of a cut dH product.
        self.live = sum(v > 0 for v in self.valid)
        live = self.valid[:self.live]
        sizes = []      # workspace of the ways to group the shards, the one that groups the most first; the second value: pass S too
        if all(v > 0 for v in live):
            bwd = max(nbytes, B.vp_output_group_workspace_bytes(B.VP_CALL_OUTPUT_BWD, N, h, live, self.dt,
                                                                flags | (B.VP_SKIP_DH if algorithm == 2 else 0)))
            try:
                sizes.append((max(bwd, B.vp_output_group_workspace_bytes(fwd_call, N, h, live, self.dt, flags)), True))
            except B.VPError:      # Algorithm 2: more shards or larger ones than one call takes
                if algorithm == 1:
                    raise
            # (Algorithm 2: pass S of all shards keeps their softmax' matrices and slices of A, pass T and the barrier need less)
            if algorithm == 2 and (not sizes or bwd < sizes[0][0]):
                sizes.append((bwd, False))
        # Algorithm 2 keeps A = softmax' W_r and B = G W_r of every shard until the barrier (A apart from one another where the
        # calls of a single shard, which take 16-byte aligned matrices, write them)
        self.Bm = [torch.empty((N, h), dtype=H.dtype, device=dev) for _ in range(p)] if algorithm == 2 else None

        def buffers(nbytes, pass_S):
            A = None
            if algorithm == 2:
                A = torch.empty((p, N, h), **f32) if pass_S else [torch.empty((N, h), **f32) for _ in range(p)]
            return torch.empty((nbytes,), dtype=torch.uint8, device=dev), A

        self.grouped = self.grouped_S = False
        for size, pass_S in sizes:
            # a single shard gains from the group calls only their K slices, which need workspace
            if (self.live == 1 and size == nbytes) or (workspace_limit is not None and size > max(nbytes, workspace_limit)):
                continue
            try:
                self.workspace, self.A = buffers(size, pass_S)
            except torch.OutOfMemoryError:
                continue
            self.grouped, self.grouped_S = True, pass_S and algorithm == 2
            break
        if not self.grouped:
            self.workspace, self.A = buffers(nbytes, False)

    # A view is made only of a shard with padding, and without a call per shard: on small workloads the host's work is what
    # bounds a step.
    def _real(self, tensors, r):
        """The real rows of shard r."""
        t, v = tensors[r], self.valid[r]
        return t if t.shape[0] == v else t[:v]

    def _live(self, tensors):
        """The real rows of the shards that have any."""
        return [t if t.shape[0] == v else t[:v] for t, v in zip(tensors, self.valid[:self.live])]

    def forward(self, stream=None) -> None:
        if self.norm is not None:
            self.norm.forward(stream)
        in_one_call = self.grouped if self.algorithm == 1 else self.grouped_S
        for r in range(self.live if in_one_call else 0, self.p):
            v = self.valid[r]
            if v == 0:     # all padding: the neutral element of the combine (exp(-inf) = 0)
                with _on(stream):
                    self.local_max[r].fill_(float("-inf"))
                    self.local_sumexp[r].zero_()
                    self.local_target[r].zero_()
                continue
            lg = self.logits[r] if self.logits is not None else None
            if self.algorithm == 1:
                B.vp_output_fwd(self.H, self._real(self.W, r), self.labels, self.offsets[r],
                                self.local_max[r], self.local_sumexp[r], self.local_target[r],
                                lg, self.workspace, stream)
            else:
                B.vp_output_fwd_alg2(self.H, self._real(self.W, r), self.labels, self.offsets[r],
                                     self.local_max[r], self.local_sumexp[r], self.local_target[r],
                                     self.A[r], self.Bm[r], lg, self.workspace, stream)
        if in_one_call:
            q = self.live
            stats = (self.local_max, self.local_sumexp, self.local_target)
            stats = stats if q == self.p else tuple(t[:q] for t in stats)
            lg = self.logits[:q] if self.logits is not None else None
            if self.algorithm == 1:
                B.vp_output_fwd_group(self.H, self._live(self.W), self.labels, self.offsets[:q], *stats, lg, self.workspace,
                                      stream)
            else:
                B.vp_output_fwd_alg2_group(self.H, self._live(self.W), self.labels, self.offsets[:q], *stats, self.A[:q],
                                           self.Bm[:q], lg, self.workspace, stream)
        B.vp_combine_stats(self.local_max, self.local_sumexp, self.local_target,
                           self.global_max, self.global_sumexp, self.loss_rows, self.loss, stream)
        if self.algorithm == 2:
            # still inside the one barrier of Algorithm 2: the input gradient leaves here; the first shard
            # that contributes overwrites dH, so nothing is zero-filled
            first = True
            if self.grouped_S:
                q = self.live
                B.vp_output_dx_alg2_gather(self.A[:q], self._live(self.W), self.labels, self.offsets[:q], self.local_max[:q],
                                           self.local_sumexp[:q], self.global_max, self.global_sumexp, self.grad_scale,
                                           self.dH, stream, dh_overwrite=True)
                return
            if self.grouped:
                q = self.live
                B.vp_output_dx_alg2_group(self.A[:q], self.Bm[:q], self.local_max[:q], self.local_sumexp[:q],
                                          self.global_max, self.global_sumexp, self.grad_scale, self.dH, stream,
                                          dh_overwrite=True)
                return
            for r in range(self.p):
                if self.valid[r] > 0:
                    B.vp_output_dx_alg2(self.A[r], self.Bm[r], self.local_max[r], self.local_sumexp[r],
                                        self.global_max, self.global_sumexp, self.grad_scale, self.dH, stream,
                                        dh_overwrite=first)
                    first = False
            if first:      # no shard holds a real vocabulary row (cannot happen: vocab_size > 0)
                with _on(stream):
                    self.dH.zero_()

    def backward(self, stream=None) -> None:
        first = True      # the first shard that contributes overwrites dH (Algorithm 1): no zero-fill
        for r in range(self.p):
            v = self.valid[r]
            if v < self.rows[r]:
                with _on(stream):
                    self.dW[r][v:].zero_()
            if v == 0 or self.grouped:
                continue
            B.vp_output_bwd(self.H, self._real(self.W, r), self.labels, self.offsets[r], self.global_max, self.global_sumexp,
                            self.logits[r] if self.logits is not None else None, self.grad_scale,
                            self.dH if self.algorithm == 1 else None, self._real(self.dW, r), self.workspace, stream,
                            dh_overwrite=first)
            first = False
        if self.grouped:
            q = self.live
            B.vp_output_bwd_group(self.H, self._live(self.W), self.labels, self.offsets[:q],
                                  self.global_max, self.global_sumexp, self.logits[:q] if self.logits is not None else None,
                                  self.grad_scale, self.dH if self.algorithm == 1 else None,
                                  self._live(self.dW), self.workspace, stream, dh_overwrite=True)
        if self.norm is not None:
            self.norm.backward(self.dH, stream=stream)

    def clip_gradients(self, max_norm: float, others: Sequence[torch.Tensor] = (), stream=None) -> torch.Tensor:
        """Clips in place by the norm of all gradients together, which it returns ([1], on the device, written by every call)."""
        grads = self.dW + (self.norm.parameter_gradients() if self.norm is not None else []) + list(others)
        if self.clip_plan is None or not self.clip_plan.covers(grads):
            # the norm and the workspaces stay where they are as long as this plan lives: a captured call has their addresses
            need = B.vp_grad_workspace_bytes(len(grads))
            with _on(stream):      # (the memory of a stream: the current one's may be in use by work before this call)
                if self.clip_norm is None:
                    self.clip_norm = torch.empty((1,), dtype=torch.float32, device=self.dH.device)
                if not self.clip_workspaces or self.clip_workspaces[-1].numel() < need:
                    self.clip_workspaces.append(torch.empty((need,), dtype=torch.uint8, device=self.dH.device))
            self.clip_plan = GradientClipPlan(grads, norm=self.clip_norm, workspace=self.clip_workspaces[-1])
        self.clip_plan.clip(max_norm, stream)
        return self.clip_norm

    def step(self, stream=None) -> None:
        self.forward(stream)
        self.backward(stream)

    def result(self) -> OutputLayerResult:
        return OutputLayerResult(self.loss, self.loss_rows, self.global_max, self.global_sumexp,
                                 self.local_max, self.local_sumexp, self.local_target,
                                 self.dH, self.dW, self.logits)


def quantize_rows(x: torch.Tensor, stream=None):
    """The rows of x in 8-bit integers, and their scales: what OutputLayerI8Plan takes for a shard of the weights.  (A shard cut from
    a larger matrix begins at any element; the library takes matrices that begin at 16 bytes, so such a one is copied.)"""
    if x.dim() != 2:
        raise B.VPError("x must be [rows, h]")
    with _on(stream):
        if x.is_contiguous() and x.data_ptr() % 16:
            x = x.clone()
        q = torch.empty((x.shape[0], B.vp_i8_row_stride(x.shape[1])), dtype=torch.int8, device=x.device)
        scales = torch.empty((x.shape[0],), dtype=torch.float32, device=x.device)
    B.vp_quantize_rows(x, q, scales, stream)
    return q, scales


class OutputLayerI8Plan:
    """The output layer's logits and statistics with weights and hidden states in 8-bit integers, for answering and scoring: there
    is no backward pass.  ``W_shards`` are pairs of integers and scales (``quantize_rows`` of a shard, made once and shared by
    plans of all sizes); the rows of H become integers in every pass.  Shards, padding (``vocab_size``) and ``norm`` are those of
    OutputLayerPlan.  Without ``labels`` loss and target logits stand for nothing.  ``logits`` are kept (``save_logits``) in
    ``logits_dtype``, by default that of H: what DraftVerifyPlan draws tokens from."""

    def __init__(self, H: Optional[torch.Tensor], W_shards, labels: Optional[torch.Tensor] = None, *, save_logits: bool = True,
                 logits_dtype: Optional[torch.dtype] = None, vocab_size: Optional[int] = None,
                 norm: Optional[BlockNormPlan] = None):
        if (H is None) == (norm is None):
            raise B.VPError("either H or the norm that makes it")
        H = norm.H if H is None else H
        if H.dim() != 2:
            raise B.VPError("H must be [N, h]")
        W_shards = list(W_shards)
        self.H, self.norm = H, norm
        self.N, self.h = H.shape
        stride = B.vp_i8_row_stride(self.h)
        offset, total = 0, sum(int(q.shape[0]) for q, _ in W_shards)
        self.vocab_size = total if vocab_size is None else int(vocab_size)
        if not 0 < self.vocab_size <= total:
            raise B.VPError("vocab_size must be in (0, total rows]")
        self.W, self.W_scales, self.offsets, self.valid = [], [], [], []      # of the shards with real rows
        for q, scales in W_shards:
            rows, valid = int(q.shape[0]), max(0, min(int(q.shape[0]), self.vocab_size - offset))
            if q.dim() != 2 or q.shape[1] != stride or scales.shape != (rows,):
                raise B.VPError("every shard must be ([rows, %d] integers, [rows] scales)" % stride)
            if valid > 0:
                self.W.append(q if valid == rows else q[:valid])
                self.W_scales.append(scales if valid == rows else scales[:valid])
                self.offsets.append(offset)
                self.valid.append(valid)
            offset += rows
        self.p = len(self.W)
        dev = H.device
        f32 = dict(dtype=torch.float32, device=dev)
        self.labels = torch.full((self.N,), -1, dtype=torch.int64, device=dev) if labels is None else labels
        self.H_i8 = torch.empty((self.N, stride), dtype=torch.int8, device=dev)
        self.H_scales = torch.empty((self.N,), **f32)
        self.local_max, self.local_sumexp, self.local_target = (torch.empty((self.p, self.N), **f32) for _ in range(3))
        self.global_max, self.global_sumexp, self.loss_rows = (torch.empty((self.N,), **f32) for _ in range(3))
        self.loss = torch.empty((1,), **f32)
        self.logits = ([torch.empty((self.N, v), dtype=logits_dtype or H.dtype, device=dev) for v in self.valid]
                       if save_logits else None)
        self.workspace = torch.empty((B.vp_output_i8_workspace_bytes(self.N, self.valid),), dtype=torch.uint8, device=dev)

    def forward(self, stream=None) -> None:
        if self.norm is not None:
            self.norm.forward(stream)
        B.vp_quantize_rows(self.H, self.H_i8, self.H_scales, stream)
        B.vp_output_fwd_i8_group(self.H_i8, self.H_scales, self.W, self.W_scales, self.labels, self.offsets, self.local_max,
                                 self.local_sumexp, self.local_target, self.logits, self.workspace, stream)
        B.vp_combine_stats(self.local_max, self.local_sumexp, self.local_target, self.global_max, self.global_sumexp,
                           self.loss_rows, self.loss, stream)


class KeptLogits:
    """The logits that a plan keeps, as DraftVerifyPlan reads them, and their statistics ``global_max`` and ``global_sumexp``: those
    of exactly the values that are stored.  (The plan's own are taken before the logits are rounded to bf16, and before the program
    changes them.)  Whatever else is asked for is the plan's."""

    def __init__(self, plan):
        if plan.logits is None:
            raise B.VPError("plans whose logits are drawn from keep them (save_logits)")
        live = [r for r, v in enumerate(plan.valid) if v > 0]
        self.plan = plan
        self.logits, self.offsets = [plan.logits[r] for r in live], [plan.offsets[r] for r in live]
        rows = [int(t.shape[1]) for t in self.logits]
        self.global_max, self.global_sumexp = (torch.empty((plan.N,), dtype=torch.float32, device=self.logits[0].device)
                                               for _ in range(2))
        self.stats_workspace = torch.empty((B.vp_logits_stats_workspace_bytes(plan.N, rows),), dtype=torch.uint8,
                                           device=self.logits[0].device)

    def __getattr__(self, name):
        if name == "plan":      # (not made yet)
            raise AttributeError(name)
        return getattr(self.plan, name)

    def statistics(self, stream=None) -> None:
        B.vp_logits_stats(self.logits, self.global_max, self.global_sumexp, self.stats_workspace, stream)


class DraftVerifyPlan:
    """Verification of drafted tokens against the logits that ``target`` keeps (an OutputLayerPlan or OutputLayerI8Plan), and the
    draw of the token behind them.  Sequence b has the rows starts[b] .. starts[b + 1] - 1 of the target's tokens, one for each
    of its drafts and a last one; ``drafts`` [N] holds the token that each row is asked about, ``uniforms`` [N] random numbers in
    [0, 1).  ``draft``: the plan of the model that drew the drafts, with the same shards and rows (its last rows stand for
    nothing), or None.  Tokens follow softmax of the logits as they are stored when ``forward`` is called: before it a program
    may rule tokens out in them (-inf) or divide them by a temperature.  Results: ``accepted`` [sequences], ``tokens`` [N]."""

    def __init__(self, target, starts: torch.Tensor, drafts: torch.Tensor, uniforms: torch.Tensor, draft=None):
        if starts.dim() != 1:
            raise B.VPError("starts must be [sequences + 1]")
        self.target, self.draft = KeptLogits(target), None if draft is None else KeptLogits(draft)
        self.starts, self.drafts, self.uniforms = starts, drafts, uniforms
        self.logits, self.offsets = self.target.logits, self.target.offsets
        self.draft_logits = None
        if draft is not None:
            self.draft_logits = self.draft.logits
            if self.draft.offsets != self.offsets or [t.shape for t in self.logits] != [t.shape for t in self.draft_logits]:
                raise B.VPError("the plans of the target and of the draft model have the same shards and rows")
        V, sequences = sum(int(t.shape[1]) for t in self.logits), starts.shape[0] - 1
        self.accepted = torch.empty((max(sequences, 0),), dtype=torch.int32, device=starts.device)
        self.tokens = torch.empty((target.N,), dtype=torch.int64, device=starts.device)
        self.workspace = torch.empty((B.vp_verify_workspace_bytes(sequences, V),), dtype=torch.uint8, device=starts.device)

    def forward(self, stream=None) -> None:
        t, d = self.target, self.draft
        t.statistics(stream)
        if d is not None:
            d.statistics(stream)
        B.vp_verify_drafts(self.logits, self.offsets, t.global_max, t.global_sumexp, self.drafts, self.starts,
                           self.uniforms, self.accepted, self.tokens, self.workspace, draft_logits=self.draft_logits,
                           draft_max=None if d is None else d.global_max, draft_sumexp=None if d is None else d.global_sumexp,
                           stream=stream)


def output_layer_step(H, W_shards, labels, save_logits=True, grad_scale=None, vocab_size=None) -> OutputLayerResult:
    """One forward + backward of the sharded output layer; returns all outputs."""
    plan = OutputLayerPlan(H, W_shards, labels, save_logits, grad_scale, vocab_size)
    plan.step()
    return plan.result()


class EmbeddingPlan:
    """Buffers and launch order for the sharded input layer (appendix C)."""

    def __init__(self, table_shards: List[torch.Tensor], ids: torch.Tensor, grad_out: Optional[torch.Tensor]):
        self.tables, self.ids, self.grad_out = table_shards, ids, grad_out
        self.p = len(table_shards)
        self.Vs, self.h = table_shards[0].shape
        self.N = ids.shape[0]
        dev = ids.device
        self.dt = B.VP_F32 if table_shards[0].dtype == torch.float32 else B.VP_BF16
        self.out = [torch.empty((self.N, self.h), dtype=table_shards[0].dtype, device=dev) for _ in range(self.p)]
        self.dtable = [torch.zeros((self.Vs, self.h), dtype=torch.float32, device=dev) for _ in range(self.p)]
        # the gradient may be of the other type than the tables, and the size depends on it
        nbytes = max([256] + [B.vp_workspace_bytes(B.VP_CALL_EMBED_BWD, self.N, self.h, self.Vs, dt, 0)
                              for dt in (B.VP_F32, B.VP_BF16)])
        self.workspace = torch.empty((nbytes,), dtype=torch.uint8, device=dev)

    def forward(self, stream=None) -> None:
        if self.p > 1 and B.same_shapes(self.tables):
            B.vp_embed_fwd_group(self.tables, self.ids, 0, self.out, stream)
            return
        for r in range(self.p):       # a single shard (the group call costs the host 1 us more), shards of different sizes
            B.vp_embed_fwd(self.tables[r], self.ids, r * self.Vs, self.out[r], stream)

    def backward(self, stream=None) -> None:
        if self.p == 1:
            B.vp_embed_bwd(self.grad_out, self.ids, 0, self.dtable[0], self.workspace, stream)
            return
        B.vp_embed_bwd_group(self.grad_out, self.ids, 0, self.dtable, self.workspace, stream)


def embedding_forward(table_shards, ids):
    plan = EmbeddingPlan(table_shards, ids, None)
    plan.forward()
    return plan.out


def _disjoint(tensors) -> bool:
    """Whether no two of the (contiguous) tensors share memory: one launch writes all of them in no order."""
    spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in tensors)
    return all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))


def embedding_backward(grad_out, ids, Vs: int, p: int, dtable: Optional[List[torch.Tensor]] = None):
    """Scatter-add into (optionally supplied, accumulate-into) fp32 shard gradients."""
    N, h = grad_out.shape
    dev = grad_out.device
    if dtable is None:
        dtable = [torch.zeros((Vs, h), dtype=torch.float32, device=dev) for _ in range(p)]
    dt = B.VP_F32 if grad_out.dtype == torch.float32 else B.VP_BF16
    used = [dtable[r] for r in range(p)]
    nbytes = max([256] + [B.vp_workspace_bytes(B.VP_CALL_EMBED_BWD, N, h, int(d.shape[0]), dt, 0) for d in used])
    ws = torch.empty((nbytes,), dtype=torch.uint8, device=dev)
    if used and all(d.shape[0] == Vs for d in used) and _disjoint(used):
        B.vp_embed_bwd_group(grad_out, ids, 0, used, ws)
        return dtable
    for r in range(p):       # gradients of other sizes, or that share memory: one after the other
        B.vp_embed_bwd(grad_out, ids, r * Vs, dtable[r], ws)
    return dtable
