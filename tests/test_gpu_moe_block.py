"""The MoE block that runs the operators together, and MXFP8 token rows in
streamFFN."""
import numpy as np
import pytest
import torch

from oracle import mx
from paper_2609_33252_amd import cep, moe_block, workload as W

from . import _block_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cep.lib()
    torch.cuda.set_device(0)


def _block(seed, ranks, rank, d=256, d_ff=128, d_shared=200, E=8, k=3, T=300):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s, std=0.05: torch.randn(*s, device="cuda", generator=g).mul_(std).bfloat16()
    experts = [n(E, d, d_ff), n(E, d, d_ff), n(E, d_ff, d)]
    shared = (n(d, d_shared), n(d, d_shared), n(d_shared, d))
    norm = 1 + 0.1 * torch.randn(d, device="cuda", generator=g)
    gate = torch.randn(d, E, device="cuda", generator=g).mul_(0.1)
    per = E // ranks
    mine = [w[rank * per:(rank + 1) * per].contiguous() for w in experts]
    b = moe_block.MoEBlock(d=d, d_ff=d_ff, d_shared=d_shared, n_experts=E, top_k=k,
                           n_ranks=ranks, rank=rank, max_tokens=T, norm=norm, gate=gate,
                           shared=shared, experts=cep.make_weights(*mine), w_dtype=cep.CEP_BF16)
    return b, experts, n


@pytest.mark.parametrize("ranks,rank", [(1, 0), (4, 1)])
def test_block_matches_its_definition(ranks, rank):
    b, experts, n = _block(ranks, ranks, rank)
    per = 8 // ranks
    for T, xt in ((1, torch.bfloat16), (77, torch.float32), (300, torch.bfloat16)):
        x, res = n(T, b.d, std=1.0).to(xt), n(T, b.d, std=1.0)
        s, y = R.rms_norm(x, res, b.norm, moe_block.EPS)
        y = y.bfloat16()
        out = b.forward(x, res)
        torch.cuda.synchronize()
        cep.cep_get_status(b.ctx)
        assert torch.equal(res, s.bfloat16())
        # the block's own choice: its logits come from a float32 product
        ids, w = b.ids[:T].long(), b.w[:T].double()
        rid, rw = R.gate((b.y[:T].float() @ b.gate).cpu().numpy(), b.top_k)
        assert np.array_equal(ids.cpu().numpy(), rid)
        ref = R.gated_ffn(b.y[:T], *b.shared)[3]
        for e in range(rank * per, (rank + 1) * per):
            wt = torch.where(ids == e, w, 0.0).sum(1, keepdim=True)
            ref = ref + wt * R.gated_ffn(b.y[:T], *(t[e] for t in experts))[3]
        # y within bf16 of the norm; the experts' outputs within their own
        # documented bounds (bf16 hidden rows)
        assert ((b.y[:T].double() - y.double()).abs() <= 2.0 ** -7 * y.double().abs()).all()
        err = (out.double() - ref).norm() / ref.norm()
        assert err < 5e-3, (T, float(err))
    b.close()


def test_block_with_e4m3_experts_takes_mxfp8_rows():
    d, I, E, k, T = 512, 256, 8, 2, 200
    wl = W.generate("fp8_fetch_d6144", 0, d=d, I=I, E=E, Eg=E, k=k, R=1, T=16, cpr=1)
    g = torch.Generator(device="cuda").manual_seed(4)
    n = lambda *s, std=0.05: torch.randn(*s, device="cuda", generator=g).mul_(std).bfloat16()
    keep = [t.cuda() for t in (wl.w_gate, wl.w_up, wl.w_down, wl.s_gate, wl.s_up, wl.s_down)]
    b = moe_block.MoEBlock(d=d, d_ff=I, d_shared=64, n_experts=E, top_k=k, n_ranks=1, rank=0,
                           max_tokens=T, norm=torch.ones(d, device="cuda"),
                           gate=torch.randn(d, E, device="cuda", generator=g),
                           shared=(n(d, 64), n(d, 64), n(64, d)),
                           experts=cep.make_weights(*keep), w_dtype=cep.CEP_FP8_E4M3_B128)
    out = b.forward(n(T, d, std=1.0), n(T, d, std=1.0))
    torch.cuda.synchronize()
    cep.cep_get_status(b.ctx)
    value = lambda q, s: (q.view(torch.float8_e4m3fn).double()
                          * s.double().repeat_interleave(128, 1).repeat_interleave(128, 2))
    wg, wu, wd = (value(q, s) for q, s in zip(keep[:3], keep[3:]))
    ref = R.gated_ffn(b.y, *b.shared)[3]
    for e in range(E):
        wt = torch.where(b.ids == e, b.w.double(), 0.0).sum(1, keepdim=True)
        ref = ref + wt * R.gated_ffn(b.y, wg[e], wu[e], wd[e])[3]
    # the bound of e4m3 experts, whose rows and hidden rows are 8-bit
    assert (out.double() - ref).norm() / ref.norm() < 4e-2
    b.close()


def test_block_gradients():
    b, _, n = _block(9, 1, 0)
    T = 130
    x, res, dout, dres = (n(T, b.d, std=1.0) for _ in range(4))
    b.forward(x, res, train=True)
    dx, d_norm, dw = b.backward(dout, dres)
    y = b.y[:T].clone()
    ref = R.gated_ffn_grad(dout, y, *b.shared)
    rx, rw = R.rms_norm_grad(res, b.norm, ref["dx"], dres, moe_block.EPS)
    for got, want in ((dx, rx), (d_norm, rw), (dw[0], ref["dwg"]), (dw[1], ref["dwu"]),
                      (dw[2], ref["dwd"])):
        # at most three bf16 roundings of random signs on the way: 3 * 2^-8 / 3^.5
        assert (got.double() - want).norm() / want.norm() < 3 * 2.0 ** -8 / 3 ** 0.5
    b.close()


def test_block_refuses_more_tokens_than_it_holds():
    b, _, n = _block(3, 1, 0, T=16)
    with pytest.raises(ValueError):
        b.forward(n(17, b.d), n(17, b.d))
    b.close()


def _layer(wl, x_dtype, rows_of, policy, theta=1):
    """One layer of workload wl with rows in x_dtype: rows_of(x) -> a tensor."""
    c = wl.cfg
    cfg = cep.make_config(d_model=c["d"], d_ff=c["I"], n_local_experts=c["E"], top_k=c["k"],
                          max_replicas=c["R"], max_tokens_per_replica=c["T"],
                          w_dtype={W.FP8: cep.CEP_FP8_E4M3_B128, W.MXFP4: cep.CEP_MXFP4}[c["w"]],
                          x_dtype=x_dtype, n_streams=2)
    keep = [t.cuda() for t in (wl.w_gate, wl.w_up, wl.w_down, wl.s_gate, wl.s_up, wl.s_down)]
    ctx = cep.cep_init_experts(cfg, cep.make_weights(*keep), None, None)
    out = torch.zeros(c["R"], c["T"], c["d"], device="cuda")
    per = [0] * c["R"]
    for ch in wl.chunks:
        per[ch.replica] += 1
    cep.cep_set_policy(ctx, policy, theta, 2)
    cep.cep_begin_layer(ctx, 1, per, out)
    for ch in wl.chunks:
        x, ids, w = wl.chunk_rows(ch)
        a = [torch.from_numpy(ch.token_idx.astype(np.int32)).cuda(), rows_of(x),
             torch.from_numpy(np.ascontiguousarray(ids, np.int32)).cuda(),
             torch.from_numpy(np.ascontiguousarray(w, np.float32)).cuda()]
        keep.append(a)
        torch.cuda.synchronize()
        cep.cep_submit_chunk(ctx, 1, ch.replica, ch.n_rows, int((ids >= 0).sum()), *a, None)
    cep.cep_combine(ctx, None)
    torch.cuda.synchronize()
    cep.cep_get_status(ctx)
    cep.cep_destroy(ctx)
    return out


def _mxfp8_rows(x):
    codes, scodes = mx.quantize_mxfp8(x.float().numpy())
    n, d = x.shape
    rows = np.zeros((n, cep.cep_row_bytes(d, cep.CEP_MXFP8)), np.uint8)
    rows[:, :d] = codes.reshape(n, d)
    rows[:, d:d + d // 32] = scodes.reshape(n, -1)
    return torch.from_numpy(rows).cuda()


@pytest.mark.parametrize("name,over,policy", [
    ("mxfp4_dsv4flash_d4096", dict(d=256, I=128, E=8, Eg=16, R=2, T=256, cpr=2), cep.CEP_PER_CHUNK),
    # 20 K pairs in one batch: the pack with the scale layout in a launch of its own
    ("mxfp4_dsv4flash_d4096", dict(d=512, I=256, E=8, Eg=8, R=2, T=1700, cpr=1), cep.CEP_WAIT_ALL),
    ("fp8_fetch_d6144", dict(d=768, I=256, E=8, Eg=16, R=2, T=300, cpr=1),
     cep.CEP_WAIT_ALL),
])
def test_mxfp8_rows_give_the_bits_of_bf16_rows(name, over, policy):
    # the library quantises bf16 rows to the same codes and scales
    wl = W.generate(name, 0, **over)
    a = _layer(wl, cep.CEP_BF16, lambda x: x.cuda(), policy)
    b = _layer(wl, cep.CEP_MXFP8, _mxfp8_rows, policy)
    assert torch.equal(a, b) and a.abs().sum() > 0


def test_mxfp8_rows_need_quantised_experts():
    base = dict(d_model=256, d_ff=128, n_local_experts=8, top_k=2, max_replicas=1,
                max_tokens_per_replica=16, n_streams=1, x_dtype=cep.CEP_MXFP8)
    for w in (cep.CEP_F32, cep.CEP_BF16):
        assert cep.cep_packed_expert_bytes(cep.make_config(w_dtype=w, **base)) == 0
    for w in (cep.CEP_FP8_E4M3_B128, cep.CEP_MXFP4):
        assert cep.cep_packed_expert_bytes(cep.make_config(w_dtype=w, **base)) > 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_block_gradients_of_every_path(dtype):
    """With the gradient of y along the routed experts and the gate, the block's
    gradients are those of its output: differentiated here as a whole, from the
    updated residual, in float64."""
    b, experts, n = _block(11, 1, 0)
    T = 90
    x, res, dout, dres = (n(T, b.d, std=1.0) for _ in range(4))
    b.forward(x, res, train=True)
    ids = b.ids[:T].long()

    def routed(y):  # coefficients: the softmax over the chosen
        w = torch.softmax((y @ b.gate.double()).gather(1, ids), 1)
        out = torch.zeros_like(y)
        for e in range(8):
            at = torch.where(ids == e, w, 0.0).sum(1, keepdim=True)
            out = out + at * R.gated_ffn(y, *(t[e] for t in experts))[3]
        return out

    y = b.y[:T].double().requires_grad_()
    d_y, = torch.autograd.grad((routed(y) * dout.double()).sum(), y)
    dx, d_norm, _ = b.backward(dout, dres, d_y=d_y.to(dtype))

    s, norm = res.double().requires_grad_(), b.norm.double().requires_grad_()
    y = s * torch.rsqrt((s * s).mean(-1, keepdim=True) + moe_block.EPS) * norm
    out = routed(y) + R.gated_ffn(y, *b.shared)[3]
    want = torch.autograd.grad((out * dout.double()).sum() + (s * dres.double()).sum(), (s, norm))
    for got, ref in zip((dx, d_norm), want):
        # six bf16 roundings of random signs at most: s, y, the hidden gradients,
        # dy, d_y and dx
        assert (got.double() - ref).norm() / ref.norm() < 6 * 2.0 ** -8 / 3 ** 0.5
    b.close()


def test_block_refuses_what_it_would_misread():
    b, _, n = _block(13, 1, 0, T=40)
    T, d = 24, b.d
    x, res, dout = n(T, d), n(T, d), n(T, d)
    wide = n(T, 2 * d)
    kept = wide.clone()
    for bad in (x.half(), x.double(), x[:, :d - 1], wide[:, :d], x[None], x.cpu(),
                x.t().contiguous().t()):
        with pytest.raises(ValueError, match="^x "):
            b.forward(bad, res)
    for bad in (res.float(), res.half(), wide[:, :d], res[:T - 1], res.cpu()):
        with pytest.raises(ValueError, match="residual"):
            b.forward(x, bad)
    b.forward(x, res)
    with pytest.raises(ValueError, match="train"):
        b.backward(dout)
    b.forward(x, res, train=True)
    for bad in (dout.float(), dout.half(), wide[:, :d], dout[:T - 1], dout.cpu()):
        with pytest.raises(ValueError, match="d_out"):
            b.backward(bad)
        with pytest.raises(ValueError, match="d_residual"):
            b.backward(dout, bad)
    for bad in (dout.half(), wide[:, :d], dout[:T - 1], dout.cpu()):
        with pytest.raises(ValueError, match="d_y"):
            b.backward(dout, None, bad)
    b.backward(dout, res)
    torch.cuda.synchronize()
    assert torch.equal(wide, kept)
    b.close()


@pytest.mark.parametrize("name,wrong", [
    ("norm", lambda t: t.bfloat16()), ("norm", lambda t: t[:-1]), ("gate", lambda t: t[:, :4]),
    ("gate", lambda t: t.bfloat16()), ("bias", lambda t: t.double()), ("bias", lambda t: t[:7]),
    ("bias", lambda t: t.repeat(2)[::2]), ("shared", lambda t: (t[0].float(), *t[1:])),
    ("shared", lambda t: (t[0], t[1], t[2].t())), ("shared", lambda t: t[:2])])
def test_block_refuses_weights_it_would_misread(name, wrong):
    d, I, E = 256, 128, 8
    g = torch.Generator(device="cuda").manual_seed(0)
    n = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    a = dict(norm=torch.ones(d, device="cuda"), gate=n(d, E).float(), bias=n(E).float(),
             shared=(n(d, 64), n(d, 64), n(64, d)))
    experts = [n(E, d, I), n(E, d, I), n(E, I, d)]
    a[name] = wrong(a[name])
    with pytest.raises(ValueError, match=name):
        moe_block.MoEBlock(d=d, d_ff=I, d_shared=64, n_experts=E, top_k=2, n_ranks=1, rank=0,
                           max_tokens=16, experts=cep.make_weights(*experts),
                           w_dtype=cep.CEP_BF16, score=cep.CEP_SIGMOID, **a)
