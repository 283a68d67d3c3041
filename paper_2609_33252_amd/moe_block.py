"""One MoE block on one GPU: the operators around the routed experts with them.

    residual += x;  y = rms_norm(residual)             cep_rms_norm
    experts of each token from y W_gate                cep_gate_topk
    rows packed per expert-parallel rank               cep_dispatch
    this rank's routed experts                         cep_begin_layer ... cep_combine
    shared expert on every token                       cep_gated_ffn
    out = routed + shared

With e4m3 or MXFP4 experts the norm writes the dispatched rows as MXFP8, which
the experts take as they are.  A block of an expert-parallel job sends the other
ranks' segments of the send buffer to them; here they are only packed.  The
gate's projection is a plain product and goes to the library.

``backward`` gives the gradients of the shared expert's weights, the norm's weight
and the block's input.  The streamed experts have no gradient, but y reaches the
output through them and the gate too: a program that trains the norm, or anything
before the block, passes that part of the gradient of y in.  Where one rank holds
every expert in bf16, it comes from

    RoutedExperts.forward, .backward      cep_expert_sort, cep_linear, cep_expert_unsort
    MoEBlock.gate_backward                cep_gate_topk_backward

Run ``python -m paper_2609_33252_amd.moe_block`` for a small block on cuda:0.
"""
from __future__ import annotations

import torch

from . import cep

EPS = 1e-6
MAX_ROWS = 1 << 21  # of an operator's descriptor


def _expect(name, t, device, dtypes, shape, dense=True):
    """The operators get plain pointers: t has to be what they read."""
    if (not isinstance(t, torch.Tensor) or t.device != device or t.dtype not in dtypes
            or t.shape != shape or (dense and not t.is_contiguous())):
        kinds = " or ".join(str(d).removeprefix("torch.") for d in dtypes)
        raise ValueError(f"{name} must be a {'contiguous ' if dense else ''}{kinds} tensor of "
                         f"shape {list(shape)} on {device}")


class MoEBlock:
    """weights: norm [d] and gate [d][n_experts] float32, bias (CEP_SIGMOID)
    [n_experts] float32, shared (w_gate, w_up [d][d_shared], w_down
    [d_shared][d]) bf16, experts a cep_weights of this rank's n_experts / n_ranks
    experts in w_dtype."""

    def __init__(self, *, d, d_ff, d_shared, n_experts, top_k, n_ranks, rank, max_tokens, norm,
                 gate, shared, experts, w_dtype, score=cep.CEP_SOFTMAX, bias=None, n_groups=0,
                 topk_groups=0):
        if n_experts % n_ranks or not 0 <= rank < n_ranks:
            raise ValueError("n_ranks must divide n_experts and hold rank")
        dev, F32, BF16 = norm.device, (torch.float32,), (torch.bfloat16,)
        _expect("norm", norm, dev, F32, (d,))
        _expect("gate", gate, dev, F32, (d, n_experts), dense=False)  # torch's product reads it
        if bias is not None:
            _expect("bias", bias, dev, F32, (n_experts,))
        if len(shared) != 3:
            raise ValueError("shared must hold w_gate, w_up and w_down")
        for w, shape in zip(shared, ((d, d_shared), (d, d_shared), (d_shared, d))):
            _expect("a weight of shared", w, dev, BF16, shape)
        self.d, self.top_k, self.n_ranks, self.rank = d, top_k, n_ranks, rank
        self.max_tokens, self.d_shared = max_tokens, d_shared
        self.norm, self.gate, self.shared, self.bias = norm, gate, shared, bias
        self.gate_args = dict(n_experts=n_experts, top_k=top_k, score=score, n_groups=n_groups,
                              topk_groups=topk_groups, normalize=1, scale=1.0)
        self.per_rank = n_experts // n_ranks
        quantised = w_dtype in (cep.CEP_FP8_E4M3_B128, cep.CEP_MXFP4)
        self.row_dtype = cep.CEP_MXFP8 if quantised else cep.CEP_BF16
        self.row_bytes = cep.cep_row_bytes(d, self.row_dtype)
        self.ctx = cep.cep_init_experts(
            cep.make_config(d_model=d, d_ff=d_ff, n_local_experts=self.per_rank, top_k=top_k,
                            max_replicas=1, max_tokens_per_replica=max_tokens, w_dtype=w_dtype,
                            x_dtype=self.row_dtype, n_streams=1),
            experts, None, torch.cuda.current_stream())
        T, sent = max_tokens, max_tokens * min(top_k, n_ranks)

        def buf(*shape, dtype=torch.bfloat16):
            return torch.empty(*shape, dtype=dtype, device=dev)

        self.y = buf(T, d)
        self.rows = buf(T, self.row_bytes, dtype=torch.uint8) if quantised else self.y
        self.ids, self.w = buf(T, top_k, dtype=torch.int32), buf(T, top_k, dtype=torch.float32)
        self.plan = buf(2 * n_ranks + 2, dtype=torch.int32)
        self.token = buf(sent, dtype=torch.int32)
        self.sent_ids = buf(sent, top_k, dtype=torch.int32)
        self.sent_w = buf(sent, top_k, dtype=torch.float32)
        # rows as bytes: a segment is a chunk of this rank's or another's experts
        self.sent = buf(sent, self.row_bytes, dtype=torch.uint8)
        self.routed = buf(1, T, d, dtype=torch.float32)
        self.shared_y = buf(T, d)
        self.dispatch_ws = buf(cep.cep_dispatch_workspace(self._dispatch_desc(T)),
                               dtype=torch.uint8)
        self.ffn_ws = buf(0, dtype=torch.uint8)
        self.generation = 0
        self.saved = None  # of the last forward pass, if that was a training one

    def _dispatch_desc(self, T):
        return cep.make_dispatch(rows=T, top_k=self.top_k, n_ranks=self.n_ranks,
                                 experts_per_rank=self.per_rank, capacity=self.token.numel(),
                                 row_bytes=self.row_bytes)

    def _ffn_space(self, desc, backward):
        need = cep.cep_gated_ffn_workspace(desc, backward)
        if self.ffn_ws.numel() < need:  # grows to the largest call's
            self.ffn_ws = torch.empty(need, dtype=torch.uint8, device=self.y.device)
        return self.ffn_ws

    def forward(self, x, residual, train=False):
        """x [T][d] (float32 or bf16: the block before's output), residual [T][d]
        bf16, updated in place; both contiguous.  Returns this rank's part of the
        block's output, float32 [T][d], valid until the next call."""
        T, d, s = x.shape[0], self.d, torch.cuda.current_stream()
        if T > self.max_tokens:
            raise ValueError(f"{T} tokens, the block holds {self.max_tokens}")
        _expect("x", x, self.y.device, (torch.float32, torch.bfloat16), (T, d))
        _expect("residual", residual, self.y.device, (torch.bfloat16,), (T, d))
        self.saved = None  # a pass that fails keeps nothing
        mx = self.row_dtype == cep.CEP_MXFP8
        desc = cep.make_norm(rows=T, d=d, res_dtype=cep.CEP_BF16, w_dtype=cep.CEP_F32,
                             x_dtype=cep.CEP_F32 if x.dtype == torch.float32 else cep.CEP_BF16,
                             y_dtype=cep.CEP_BF16, eps=EPS, ld_codes=self.row_bytes if mx else 0,
                             ld_scales=self.row_bytes if mx else 0)
        cep.cep_rms_norm(desc, x, self.norm, residual=residual, res_out=residual, y=self.y,
                         codes=self.rows if mx else None,
                         scales=self.rows.data_ptr() + d if mx else None, stream=s)
        y = self.y[:T]
        logits = y.float() @ self.gate
        cep.cep_gate_topk(cep.make_gate(rows=T, **self.gate_args), logits, self.bias, self.ids,
                          self.w, stream=s)
        cep.cep_dispatch(self._dispatch_desc(T), self.ids, self.w, self.rows, self.plan,
                         self.token, self.sent_ids, self.sent_w, self.sent, self.dispatch_ws,
                         stream=s)
        # the shared expert is enqueued before the host waits for the plan
        ffn = cep.make_gated_ffn(rows=T, d_model=d, d_ff=self.d_shared)
        pre = torch.empty(T, 2, self.d_shared, device=y.device) if train else None
        cep.cep_gated_ffn(ffn, y, *self.shared, self.shared_y, self._ffn_space(ffn, train),
                          preact=pre, stream=s)
        saved = (residual.clone(), y.clone(), pre, logits, self.ids[:T].clone()) if train else None
        routed = self.routed[0, :T]
        routed.zero_()
        plan = self.plan.cpu()
        r, R = self.rank, self.n_ranks
        a, b, pairs = int(plan[r]), int(plan[r + 1]), int(plan[R + 1 + r])
        if int(plan[2 * R + 1]):
            raise RuntimeError("expert ids that no rank holds")
        self.generation += 1
        cep.cep_begin_layer(self.ctx, self.generation, [1], self.routed)
        if b > a:
            ready = torch.cuda.Event()
            ready.record(s)
            cep.cep_submit_chunk(self.ctx, self.generation, 0, b - a, pairs, self.token[a:b],
                                 self.sent[a:b], self.sent_ids[a:b], self.sent_w[a:b], ready)
        else:
            cep.cep_submit_chunk(self.ctx, self.generation, 0, 0, 0, None, None, None, None, None)
        cep.cep_combine(self.ctx, s)
        self.saved = saved
        return routed.add_(self.shared_y[:T])

    def backward(self, d_out, d_residual=None, d_y=None):
        """Gradients of a forward(train=True): d_out bf16 [T][d] of the output,
        d_residual (bf16 or None) of the updated residual, d_y (float32, bf16 or
        None) what the paths of y through the routed experts and the gate add to
        the gradient of y = ``self.y[:T]``.  Returns d_x (bf16, also the
        residual's), d_norm, and the shared expert's three weight gradients.
        d_x and d_norm are the output's gradients if d_y is complete; without it
        they leave those paths out, as one addend of the gradients."""
        if self.saved is None:
            raise ValueError("backward without a forward(train=True) before it")
        residual, y, pre, *_ = self.saved
        T, d, s = y.shape[0], self.d, torch.cuda.current_stream()
        BF16 = (torch.bfloat16,)
        _expect("d_out", d_out, y.device, BF16, (T, d))
        if d_residual is not None:
            _expect("d_residual", d_residual, y.device, BF16, (T, d))
        if d_y is not None:
            _expect("d_y", d_y, y.device, BF16 + (torch.float32,), (T, d))
        ffn = cep.make_gated_ffn(rows=T, d_model=d, d_ff=self.d_shared)
        dy = torch.empty_like(y)
        dw = [torch.empty_like(w) for w in self.shared]
        cep.cep_gated_ffn_backward(ffn, d_out, y, *self.shared, pre, dy, *dw,
                                   self._ffn_space(ffn, True), stream=s)
        if d_y is not None:
            dy = dy.float().add_(d_y)  # not rounded again
        desc = cep.make_norm(rows=T, d=d, x_dtype=cep.CEP_BF16, res_dtype=cep.CEP_BF16,
                             w_dtype=cep.CEP_F32, eps=EPS,
                             y_dtype=cep.CEP_BF16 if d_y is None else cep.CEP_F32)
        ws = torch.empty(cep.cep_rms_norm_workspace(desc), dtype=torch.uint8, device=y.device)
        dx, d_norm = torch.empty_like(y), torch.empty_like(self.norm)
        cep.cep_rms_norm_backward(desc, residual, self.norm, dy, d_residual, dx, d_norm, ws,
                                  stream=s)
        return dx, d_norm, dw

    def gate_backward(self, d_topk_w):
        """Gradients through the gate of a forward(train=True), from that of its
        coefficients, float32 [T][top_k]: of y (float32 [T][d], an addend of
        ``backward``'s d_y) and of the gate's weight (float32 [d][n_experts])."""
        if self.saved is None:
            raise ValueError("gate_backward without a forward(train=True) before it")
        _, y, _, logits, ids = self.saved
        T = y.shape[0]
        _expect("d_topk_w", d_topk_w, y.device, (torch.float32,), (T, self.top_k))
        d_logits = torch.empty_like(logits)
        cep.cep_gate_topk_backward(cep.make_gate(rows=T, **self.gate_args), logits, ids,
                                   d_topk_w, d_logits, stream=torch.cuda.current_stream())
        return d_logits @ self.gate.T, y.float().T @ d_logits

    def close(self):
        if self.ctx:
            cep.cep_destroy(self.ctx)
            self.ctx = None


class RoutedExperts:
    """Gated experts of one rank with gradients: w_gate, w_up [n_experts][d][d_ff] and
    w_down [n_experts][d_ff][d], bf16.

        sorted rows x of each expert       cep_expert_sort
        u = x W_up, h = silu(x W_gate) u   cep_linear
        h W_down, weighted and summed      cep_linear, cep_expert_unsort

    What a product reads is bf16, rounded once: x, u and h, and in the backward pass the
    gradients of the experts' rows, of h, u and z; the experts' rows before they are
    weighted too.  Sums (a token's rows, the gradient of x, of w) are float32, and z is
    kept so.
    """

    def __init__(self, *, top_k, w_gate, w_up, w_down):
        BF16 = (torch.bfloat16,)
        if w_gate.dim() != 3:
            raise ValueError("w_gate must be of shape [n_experts, d, d_ff]")
        E, d, d_ff = w_gate.shape
        _expect("w_gate", w_gate, w_gate.device, BF16, (E, d, d_ff))
        _expect("w_up", w_up, w_gate.device, BF16, (E, d, d_ff))
        _expect("w_down", w_down, w_gate.device, BF16, (E, d_ff, d))
        if not 1 <= E <= 1024 or not 1 <= top_k <= 16:
            raise ValueError("RoutedExperts holds 1 to 1024 experts, top_k of 1 to 16")
        if any(n % 8 or not 8 <= n <= 32768 for n in (d, d_ff)):
            raise ValueError("d and d_ff must be multiples of 8, up to 32768")
        self.E, self.d, self.d_ff, self.top_k = E, d, d_ff, top_k
        self.w_gate, self.w_up, self.w_down = w_gate, w_up, w_down
        self.saved = None  # of the last forward pass, if that was a training one
        self.bad_ids = None  # of the last forward pass

    def _buf(self, *shape, dtype=torch.bfloat16):
        return torch.empty(*shape, dtype=dtype, device=self.w_gate.device)

    def _space(self, need):  # the allocator's, so that calls on two streams have one each
        return self._buf(need, dtype=torch.uint8)

    def _linear(self, rows, d_in, d_out, act=cep.CEP_IDENTITY, dx_dtype=cep.CEP_BF16):
        return cep.make_linear(rows=rows, d_in=d_in, d_out=d_out, n_groups=self.E, act=act,
                               y_dtype=cep.CEP_BF16, dx_dtype=dx_dtype, dw_dtype=cep.CEP_BF16)

    def _unsort(self, T, ys_dtype, y_dtype):
        return cep.make_expert_unsort(rows=T, top_k=self.top_k, d=self.d,
                                      sorted_rows=T * self.top_k, ys_dtype=ys_dtype,
                                      y_dtype=y_dtype)

    def forward(self, y, ids, w, train=False):
        """y [T][d] bf16; ids int32 and w float32 [T][top_k] as cep_gate_topk leaves
        them (-1: empty slot).  Returns float32 [T][d], each token's weighted sum.
        Raises for ids outside [-1, n_experts), whose number is also left in
        ``bad_ids`` (int32 [1] on the device): a pass that is captured into a graph
        cannot raise, and its replays count such slots as empty."""
        T, k, d, dev = y.shape[0], self.top_k, self.d, self.w_gate.device
        _expect("y", y, dev, (torch.bfloat16,), (T, d))
        _expect("ids", ids, dev, (torch.int32,), (T, k))
        _expect("w", w, dev, (torch.float32,), (T, k))
        if T * k > MAX_ROWS:
            raise ValueError(f"{T} tokens of {k} slots: the products take up to 2^21 rows")
        self.saved = None  # a pass that fails keeps nothing
        with torch.cuda.device(dev):
            return self._forward(y, ids, w, train)

    def _forward(self, y, ids, w, train):
        T, k, d, I = y.shape[0], self.top_k, self.d, self.d_ff
        s, P = torch.cuda.current_stream(), T * k
        sort = cep.make_expert_sort(rows=T, top_k=k, n_experts=self.E, capacity=P, row_bytes=2 * d)
        plan, pair = self._buf(self.E + 2, dtype=torch.int32), self._buf(P, dtype=torch.int32)
        place, x = self._buf(T, k, dtype=torch.int32), self._buf(P, d)
        cep.cep_expert_sort(sort, ids, plan, pair, place,
                            self._space(cep.cep_expert_sort_workspace(sort)), x=y, out_x=x,
                            stream=s)
        self.bad_ids, count = plan[self.E + 1:], None
        if not torch.cuda.is_current_stream_capturing():
            # the host waits for the sort alone, with the products already enqueued
            count, sorted_ = torch.empty(1, dtype=torch.int32, pin_memory=True), torch.cuda.Event()
            count.copy_(self.bad_ids, non_blocking=True)
            sorted_.record(s)
        up, gate = self._linear(P, d, I), self._linear(P, d, I, cep.CEP_SILU)
        down = self._linear(P, I, d)
        ws = self._space(max(cep.cep_linear_workspace(q) for q in (up, gate, down)))
        u, h, out = self._buf(P, I), self._buf(P, I), self._buf(P, d)
        pre = self._buf(P, I, dtype=torch.float32) if train else None
        cep.cep_linear(up, x, self.w_up, u, ws, offsets=plan, stream=s)
        cep.cep_linear(gate, x, self.w_gate, h, ws, mul=u, offsets=plan, preact=pre, stream=s)
        cep.cep_linear(down, h, self.w_down, out, ws, offsets=plan, stream=s)
        total = self._buf(T, d, dtype=torch.float32)
        cep.cep_expert_unsort(self._unsort(T, cep.CEP_BF16, cep.CEP_F32), out, place, total, w=w,
                              stream=s)
        if count is not None:
            sorted_.synchronize()
            if int(count):
                raise RuntimeError(f"{int(count)} expert ids outside [-1, {self.E})")
        if train:
            self.saved = plan, place, w.clone(), x, u, h, pre, out
        return total

    def backward(self, d_total):
        """Gradients of a forward(train=True) from that of its output (float32 or bf16
        [T][d]): of y (float32 [T][d]), of the coefficients (float32 [T][top_k]) and
        of w_gate, w_up and w_down (bf16)."""
        if self.saved is None:
            raise ValueError("backward without a forward(train=True) before it")
        _expect("d_total", d_total, self.w_gate.device, (torch.float32, torch.bfloat16),
                (self.saved[1].shape[0], self.d))
        with torch.cuda.device(self.w_gate.device):
            return self._backward(d_total)

    def _backward(self, d_total):
        plan, place, w, x, u, h, pre, out = self.saved
        T, P, d, I, s = place.shape[0], x.shape[0], self.d, self.d_ff, torch.cuda.current_stream()
        for t in self.saved:
            t.record_stream(s)  # it may be another one than the forward pass's
        kind = cep.CEP_F32 if d_total.dtype == torch.float32 else cep.CEP_BF16
        d_out, d_w = torch.empty_like(out), torch.empty_like(w)
        cep.cep_expert_unsort_backward(self._unsort(T, cep.CEP_BF16, kind), d_total, out, place, w,
                                       d_out, d_w, stream=s)
        # x's gradient is the sum of two products' and of k rows': float32 until it is y's (8192
        # tokens to two of eight experts of 4096 x 2048, a step: 2709 us, with bf16 rows 2627)
        up = self._linear(P, d, I, dx_dtype=cep.CEP_F32)
        gate = self._linear(P, d, I, cep.CEP_SILU, dx_dtype=cep.CEP_F32)
        down = self._linear(P, I, d)
        ws = self._space(max(cep.cep_linear_workspace(q, True) for q in (up, gate, down)))
        dh, du, dx = torch.empty_like(h), torch.empty_like(u), self._buf(P, d, dtype=torch.float32)
        dw = [torch.empty_like(t) for t in (self.w_gate, self.w_up, self.w_down)]
        cep.cep_linear_backward(down, d_out, h, self.w_down, ws, dx=dh, dw=dw[2], offsets=plan,
                                stream=s)
        cep.cep_linear_backward(gate, dh, x, self.w_gate, ws, dx=dx, dw=dw[0], preact=pre, mul=u,
                                dmul=du, offsets=plan, stream=s)
        cep.cep_linear_backward(up, du, x, self.w_up, ws, dx=dx, dw=dw[1], dx_add=dx, offsets=plan,
                                stream=s)
        d_y = self._buf(T, d, dtype=torch.float32)
        cep.cep_expert_unsort(self._unsort(T, cep.CEP_F32, cep.CEP_F32), dx, place, d_y, stream=s)
        return d_y, d_w, dw


def main():
    d, d_ff, d_shared, E, k = 1024, 512, 512, 16, 4
    g = torch.Generator(device="cuda").manual_seed(0)

    def normal(*shape, std=0.02):
        return torch.randn(*shape, device="cuda", generator=g).mul_(std).bfloat16()

    experts = [normal(E, d, d_ff), normal(E, d, d_ff), normal(E, d_ff, d)]
    block = MoEBlock(d=d, d_ff=d_ff, d_shared=d_shared, n_experts=E, top_k=k, n_ranks=1, rank=0,
                     max_tokens=2048, norm=torch.ones(d, device="cuda"),
                     gate=normal(d, E).float(),
                     shared=(normal(d, d_shared), normal(d, d_shared), normal(d_shared, d)),
                     experts=cep.make_weights(*experts), w_dtype=cep.CEP_BF16)
    routed = RoutedExperts(top_k=k, w_gate=experts[0], w_up=experts[1], w_down=experts[2])
    for T in (1, 100, 2048):
        x, residual, d_out = normal(T, d, std=1.0), normal(T, d, std=1.0), normal(T, d)
        out = block.forward(x, residual, train=True)
        # the gradient through the routed experts and the gate, then all of it
        routed.forward(block.y[:T], block.ids[:T], block.w[:T], train=True)
        d_y, d_w, _ = routed.backward(d_out)
        d_gate_y, d_gate = block.gate_backward(d_w)
        dx, d_norm, _ = block.backward(d_out, d_y=d_y + d_gate_y)
        torch.cuda.synchronize()
        print(f"{T} tokens: output rms {float(out.square().mean().sqrt()):.4f}, "
              f"{int(block.plan[1])} rows sent, gradient rms of x "
              f"{float(dx.float().square().mean().sqrt()):.6f}, of the gate "
              f"{float(d_gate.square().mean().sqrt()):.6f}")
    block.close()


if __name__ == "__main__":
    main()
