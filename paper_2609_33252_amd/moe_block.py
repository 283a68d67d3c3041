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
and the block's input.  The routed experts and the gate have no gradients of
their own here, but y reaches the output through them too: a program that trains
the norm, or anything before the block, passes that part of the gradient of y in.

Run ``python -m paper_2609_33252_amd.moe_block`` for a small block on cuda:0.
"""
from __future__ import annotations

import torch

from . import cep

EPS = 1e-6


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
        self.saved = (residual.clone(), y.clone(), pre) if train else None
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
        residual, y, pre = self.saved
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

    def close(self):
        if self.ctx:
            cep.cep_destroy(self.ctx)
            self.ctx = None


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
    for T in (1, 100, 2048):
        x, residual = normal(T, d, std=1.0), normal(T, d, std=1.0)
        out = block.forward(x, residual, train=True)
        dx, d_norm, _ = block.backward(normal(T, d))
        torch.cuda.synchronize()
        print(f"{T} tokens: output rms {float(out.square().mean().sqrt()):.4f}, "
              f"{int(block.plan[1])} rows sent, gradient rms of x through the shared expert "
              f"{float(dx.float().square().mean().sqrt()):.6f}")
    block.close()


if __name__ == "__main__":
    main()
