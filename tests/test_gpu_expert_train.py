"""The operators that train through the routed experts on the GPU against float64
forms.

Tolerances, from the formats: u16 = 2^-8 is half a unit in the last place of
bf16, u32 = 2^-24 of float32.  A float32 sum of n terms in any order is within
n u32 of the sum of the magnitudes; the ones here run over at most a few hundred
sequential terms a lane, so 2^-15 of the magnitudes is ample.  An activation or
its slope costs a handful of float32 roundings, of intermediate values up to 1 +
|z|, and an exponential whose argument's rounding, up to 88 u32 log2(e), is 2^-16
of its value.
"""
import numpy as np
import pytest
import torch

from paper_2609_33252_amd import cep

from . import _block_ref as B
from . import _train_ref as R

pytestmark = pytest.mark.gpu

U16, SUM32 = 2.0 ** -8, 2.0 ** -15
F32, BF16 = cep.CEP_F32, cep.CEP_BF16
DT = {F32: torch.float32, BF16: torch.bfloat16}
NAN = float("nan")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cep.lib()
    torch.cuda.set_device(0)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype=torch.bfloat16, std=1.0):
    return torch.randn(*shape, device="cuda", generator=g).mul_(std).to(dtype)


def _close(got, ref, tol, what):
    err = (got.double() - ref).abs()
    bad = ~(err <= tol)
    assert not bad.any(), (what, float(err.max()), int(bad.sum()), bad.nonzero()[:4].tolist())


def _padded(t, ld, fill=NAN):
    """t's rows in a buffer of row stride ld; the padding is NaN."""
    buf = torch.full((*t.shape[:-1], ld), fill, dtype=t.dtype, device=t.device)
    buf[..., :t.shape[-1]] = t
    return buf


def _round_tol(ref, mag, dtype):
    return (U16 * 1.01 * ref.abs() if dtype == BF16 else 0) + SUM32 * mag + 1e-37


def _space(n, fill=255):
    return torch.full((n,), fill, dtype=torch.uint8, device="cuda")  # 255: NaN in any type


# ------------------------------------------------------------------- sort

SORTS = [
    # T, k, E, row bytes, pad, kind of ids
    (0, 2, 4, 64, 0, "any"), (1, 1, 1, 1, 0, "any"), (1, 16, 1024, 14336, 0, "any"),
    (13, 8, 32, 14336, 0, "few"), (16, 16, 64, 17, 1, "any"), (255, 4, 5, 33, 0, "any"),
    (300, 8, 16, 1000, 24, "few"), (512, 8, 64, 272, 0, "any"),   # the last in one launch
    (513, 8, 64, 272, 0, "any"), (257, 16, 1024, 130, 6, "any"),  # more launches
    (1000, 5, 3, 16, 0, "any"), (5000, 1, 7, 2, 3, "any"), (3001, 7, 160, 4112, 0, "few"),
    (600, 8, 64, 131072, 0, "few"), (20000, 16, 1023, 8, 0, "any"),
    (4096, 8, 1, 48, 0, "any"), (4097, 8, 64, 48, 0, "one"), (4097, 2, 64, 48, 0, "none"),
    (1 << 17, 16, 300, 1, 0, "any"),
    # the counts summed by the rows' workgroups, up to both limits, and past them
    (600, 15, 511, 40, 0, "any"), (600, 15, 512, 40, 0, "any"), (1024, 16, 510, 24, 0, "few"),
    (500, 16, 511, 24, 0, "any"), (4100, 11, 80, 33, 0, "any"), (4700, 11, 80, 33, 0, "any"),
    (1025, 16, 511, 24, 0, "any"), (9000, 11, 80, 33, 0, "any"), (9400, 11, 80, 33, 0, "any"),
]


def _ids(g, T, k, E, kind):
    ids = g.integers(0, E, (T, k)).astype(np.int32)  # repeats among them
    if kind == "few":
        ids[g.random((T, k)) < 0.8] = -1
    if kind == "any":
        ids[g.random((T, k)) < 0.2] = -1
        if T > 8:
            ids[4] = -1  # a token that goes nowhere
            ids[5, 0], ids[6, 0], ids[7, 0], ids[8, 0] = E, -2, 2 ** 31 - 1, -2 ** 31
    if kind == "one":
        ids[:] = E - 1
    if kind == "none":
        ids[:] = -1
    return ids


@pytest.mark.parametrize("T,k,E,row,pad,kind", SORTS)
def test_sort(T, k, E, row, pad, kind):
    g = np.random.default_rng(T * 7 + row)
    ids = _ids(g, T, k, E, kind)
    x = g.integers(0, 256, (T, row + pad)).astype(np.uint8)
    cap = T * k + 3
    desc = cep.make_expert_sort(rows=T, top_k=k, n_experts=E, capacity=cap, row_bytes=row,
                                ld_x=row + pad)
    dev = lambda a: torch.from_numpy(a).cuda()
    ref_plan, ref_pair, ref_place = R.expert_sort(ids, E)
    n = len(ref_pair)
    for copy in (True, False):
        plan = torch.full((E + 3,), 9, dtype=torch.int32, device="cuda")
        pair = torch.full((cap,), -5, dtype=torch.int32, device="cuda")
        place = torch.full((T * k + 1,), -5, dtype=torch.int32, device="cuda")
        ox = torch.full((cap, row), 5, dtype=torch.uint8, device="cuda")
        ws = _space(cep.cep_expert_sort_workspace(desc))
        cep.cep_expert_sort(desc, dev(ids), plan, pair, place, ws,
                            **(dict(x=dev(x), out_x=ox) if copy else {}))
        assert np.array_equal(plan.cpu().numpy(), [*ref_plan, 9])
        pair, place = pair.cpu().numpy(), place.cpu().numpy()
        assert np.array_equal(pair[:n], ref_pair) and (pair[n:] == -5).all()
        assert np.array_equal(place[:-1].reshape(T, k), ref_place) and place[-1] == -5
        if copy:
            want = torch.from_numpy(x[ref_pair // k, :row])
            assert torch.equal(ox[:n].cpu(), want)
        assert (ox[n if copy else 0:] == 5).all()


@pytest.mark.parametrize("T,k,E", [
    # blocks' counts summed by the rows' workgroups, up to 16 blocks (8 past 256 buckets), and
    # one block more
    (1024, 16, 8), (1025, 16, 8), (1024, 16, 255), (1025, 16, 255), (512, 16, 256), (513, 16, 256),
    (512, 16, 511), (513, 16, 511), (512, 16, 512), (16384, 1, 1), (16385, 1, 1), (60000, 8, 3)])
def test_sort_with_the_counts_of_few_and_many_blocks(T, k, E):
    test_sort(T, k, E, 40, 0, "any")


# ------------------------------------------------------------------- back

UNSORTS = [
    # T, k, d, ys, residual, y, weights, pad
    (1, 1, 1, F32, None, F32, True, 0), (1, 8, 7168, BF16, BF16, BF16, True, 0),
    (9, 8, 513, BF16, F32, F32, True, 3), (7, 16, 77, BF16, BF16, BF16, True, 1),
    (70, 6, 512, F32, BF16, F32, False, 0), (300, 3, 1000, BF16, None, F32, False, 8),
    (65, 16, 2049, F32, F32, BF16, True, 0), (33, 2, 8191, F32, None, F32, True, 0),
    (5, 4, 32768, BF16, BF16, BF16, True, 0), (1030, 8, 264, BF16, BF16, BF16, True, 0),
]


def _way_back(seed, T, k, d, ys, pad):
    """Sorted rows, their places with empty slots, rows of no pair and places out of
    range among them; rows of no pair are NaN."""
    g, r = _gen(seed), np.random.default_rng(seed)
    n = T * k + 5
    place = r.permutation(n)[:T * k].reshape(T, k).astype(np.int32)
    place[r.random((T, k)) < 0.25] = -1
    if T > 4:
        place[1] = -1  # a token of no expert
        place[2, 0], place[3, 0], place[4, 0] = n, 2 ** 31 - 1, -2 ** 31
    rows = _randn(g, n, d, dtype=DT[ys])
    free = np.setdiff1d(np.arange(n), place)
    rows[torch.from_numpy(free).cuda()] = NAN
    w = torch.rand(T, k, device="cuda", generator=g) - 0.3
    place = torch.from_numpy(place).cuda()
    w[(place < 0) | (place >= n)] = NAN  # not used
    return g, n, place, w, _padded(rows, d + pad)


@pytest.mark.parametrize("T,k,d,ys,res,y,weighted,pad", UNSORTS)
def test_unsort(T, k, d, ys, res, y, weighted, pad):
    g, n, place, w, rows = _way_back(T + d, T, k, d, ys, pad)
    w = w if weighted else None
    r = None if res is None else _randn(g, T, d, dtype=DT[res], std=3.0)
    desc = cep.make_expert_unsort(rows=T, top_k=k, d=d, sorted_rows=n, ys_dtype=ys,
                                  res_dtype=F32 if res is None else res, y_dtype=y,
                                  ld_ys=d + pad, ld_res=d + 2 * pad, ld_y=d + pad)
    out = torch.full((T, d + pad), 7.0, dtype=DT[y], device="cuda")
    cep.cep_expert_unsort(desc, rows, place, out, w=w,
                          residual=None if r is None else _padded(r, d + 2 * pad))
    ref, mag = R.expert_unsort(rows[:, :d], place, w, r)
    _close(out[:, :d], ref, _round_tol(ref, mag, y), "y")
    assert (out[:, d:] == 7.0).all()
    if r is not None and res == y:  # onto the residual itself
        both = _padded(r, d + 2 * pad, 7.0)
        desc.ld_y = desc.ld_res
        cep.cep_expert_unsort(desc, rows, place, both, w=w, residual=both)
        assert torch.equal(both[:, :d], out[:, :d]) and (both[:, d:] == 7.0).all()


@pytest.mark.parametrize("T,k,d,ys,res,y,weighted,pad", UNSORTS)
def test_unsort_backward(T, k, d, ys, res, y, weighted, pad):
    g, n, place, w, rows = _way_back(T + d + 1, T, k, d, ys, pad)
    w = w if weighted else None
    dy = _randn(g, T, d, dtype=DT[y])
    desc = cep.make_expert_unsort(rows=T, top_k=k, d=d, sorted_rows=n, ys_dtype=ys, y_dtype=y,
                                  ld_ys=d + pad, ld_y=d + pad)
    dys = torch.full((n, d + pad), 7.0, dtype=DT[ys], device="cuda")
    dw = torch.full((T, k), 7.0, device="cuda")
    dyb = _padded(dy, d + pad)
    cep.cep_expert_unsort_backward(desc, dyb, rows, place, w, dys, dw)
    rdys, rdw, mag = R.expert_unsort_grad(dy, rows[:, :d], place, w)
    none = torch.isnan(rdys)
    assert (dys[:, :d][none] == 7.0).all() and (dys[:, d:] == 7.0).all()
    rdys[none] = 7.0
    _close(dys[:, :d], rdys, _round_tol(rdys, rdys.abs(), ys), "dys")
    _close(dw, rdw, SUM32 * mag, "dw")  # empty slots exactly 0
    # each output alone, and dys onto ys
    alone, dw2 = torch.full_like(dys, 7.0), torch.full_like(dw, 3.0)
    cep.cep_expert_unsort_backward(desc, dyb, None, place, w, alone, None)
    cep.cep_expert_unsort_backward(desc, dyb, rows, place, w, None, dw2)
    assert torch.equal(alone, dys) and torch.equal(dw2, dw)
    dw2.fill_(3.0)
    cep.cep_expert_unsort_backward(desc, dyb, rows, place, w, rows, dw2)
    assert torch.equal(dw2, dw) and torch.equal(rows[:, :d][~none], dys[:, :d][~none])


def test_sort_and_its_gradient_are_adjoint():
    """<sort(x), v> = <x, unsort(v)> with values of few bits, whose sums are exact."""
    T, k, E, d = 700, 6, 16, 264
    g = _gen(2)
    ids = torch.from_numpy(_ids(np.random.default_rng(2), T, k, E, "any")).cuda()
    x = torch.randint(-8, 9, (T, d), device="cuda", generator=g).bfloat16()
    v = torch.randint(-8, 9, (T * k, d), device="cuda", generator=g).bfloat16()
    sd = cep.make_expert_sort(rows=T, top_k=k, n_experts=E, capacity=T * k, row_bytes=2 * d)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    plan, pair, place, xs = i32(E + 2), i32(T * k), i32(T, k), torch.zeros_like(v)
    cep.cep_expert_sort(sd, ids, plan, pair, place, _space(cep.cep_expert_sort_workspace(sd)), x=x,
                        out_x=xs)
    ud = cep.make_expert_unsort(rows=T, top_k=k, d=d, sorted_rows=T * k, ys_dtype=BF16, y_dtype=F32)
    dx = torch.empty(T, d, device="cuda")
    cep.cep_expert_unsort(ud, v, place, dx)
    n = int(plan[E])
    assert float((xs[:n].double() * v[:n].double()).sum()) == float((x.double() * dx.double()).sum())


# ----------------------------------------------------------------- linear

LINEARS = [
    # rows, d_in, d_out, groups: one weight
    (1, 8, 8, 0), (1, 7168, 2048, 0), (2, 264, 136, 0), (16, 512, 2048, 0), (17, 1000, 504, 0),
    (32, 40, 4096, 0), (33, 16, 4096, 0), (65, 256, 128, 0), (129, 520, 72, 0),
    (300, 264, 1032, 0), (513, 512, 384, 0), (777, 2560, 1024, 0),  # shares of K
    (3001, 1544, 3080, 0), (2047, 1032, 4104, 0),                   # 256-wide tiles
    # groups: rows by the list, the first below the offsets' start
    (60, 264, 136, [0, 5, 0, 1, 17, 33, 0]), (24, 1024, 264, [3, 3, 3, 3, 3, 3, 3, 3]),
    (100, 136, 520, [90, 2, 0, 1]), (8, 264, 136, [0, 3, 0, 0, 4, 0]), (3, 8, 264, [0, 0, 3]),
    (70, 512, 256, [0, 0, 0]), (64, 8, 8, [64]),
    (80, 1032, 264, [10] * 8), (88, 1032, 264, [11] * 8),           # streamed, and past it
    (300, 264, 392, [1, 127, 0, 128, 12]), (900, 520, 264, [257, 0, 300, 1, 255, 64]),
    (2500, 264, 1032, [1300, 0, 5, 900, 200, 3]), (130, 72, 264, [1] * 130),
    (1500, 40, 264, [5] * 300), (5000, 1024, 1544, [1027, 0, 1500, 2049, 100, 200]),
]
EXTRAS = [
    # act, bias, mul, residual, y, preact, pad
    (cep.CEP_IDENTITY, False, False, None, BF16, False, 0),
    (cep.CEP_IDENTITY, True, False, BF16, BF16, True, 8),
    (cep.CEP_RELU, True, True, F32, F32, False, 8),
    (cep.CEP_SILU, False, True, None, BF16, True, 0),
    (cep.CEP_GELU, True, False, F32, F32, True, 16),
    (cep.CEP_GELU_TANH, True, True, BF16, F32, False, 0),
]


def _linear_case(rows, d, N, groups, act, bias, mul, res, pad, seed):
    """Inputs; rows of no group (three in front, some behind) are NaN."""
    g = _gen(seed)
    lead, off, live = (), None, slice(0, rows)
    if groups:
        lead = (len(groups),)
        first = min(3, rows - sum(groups))
        assert first >= 0
        off = [int(v) for v in first + np.cumsum([0, *groups])]
        live = slice(off[0], off[-1])
    c = dict(x=_randn(g, rows, d), w=_randn(g, *lead, d, N, std=d ** -0.5))
    c["bias"] = _randn(g, *lead, N, dtype=torch.float32) if bias else None
    c["mul"] = _randn(g, rows, N) if mul else None
    c["res"] = None if res is None else _randn(g, rows, N, dtype=DT[res])
    c["dy"] = _randn(g, rows, N)
    dead = torch.ones(rows, dtype=torch.bool, device="cuda")
    dead[live] = False
    for k in ("x", "mul", "res", "dy"):
        if c[k] is not None:
            c[k][dead] = NAN
    dev = None if off is None else torch.tensor(off, dtype=torch.int32, device="cuda")
    return c, off, dev, live, dead


def _desc(rows, d, N, groups, act, res, y, pad, **kw):
    return cep.make_linear(rows=rows, d_in=d, d_out=N, n_groups=len(groups) if groups else 0,
                           act=act, y_dtype=y, res_dtype=F32 if res is None else res,
                           ld_x=d + pad, ld_y=N + pad, ld_mul=N + 2 * pad, ld_res=N + pad,
                           ld_dx=d + 2 * pad, **kw)


@pytest.mark.parametrize("rows,d,N,groups", LINEARS)
@pytest.mark.parametrize("act,bias,mul,res,y,keep,pad", EXTRAS)
def test_linear(rows, d, N, groups, act, bias, mul, res, y, keep, pad):
    c, off, dev, live, dead = _linear_case(rows, d, N, groups, act, bias, mul, res, pad,
                                           rows + d + N)
    desc = _desc(rows, d, N, groups, act, res, y, pad)
    out = torch.full((rows, N + pad), 7.0, dtype=DT[y], device="cuda")
    pre = torch.full((rows, N), 7.0, device="cuda") if keep else None
    args = dict(bias=c["bias"], mul=_padded(c["mul"], N + 2 * pad) if mul else None,
                residual=None if res is None else _padded(c["res"], N + pad), offsets=dev)
    xb = _padded(c["x"], d + pad)
    ws = _space(cep.cep_linear_workspace(desc))
    cep.cep_linear(desc, xb, c["w"], out, ws, preact=pre, **args)
    z, ref, mag = R.linear(c["x"], c["w"], c["bias"], c["mul"], c["res"], act, off)
    assert (out[dead] == 7.0).all() and (out[:, N:] == 7.0).all()
    a = R.act(act, z)[0].abs()
    ez = SUM32 * mag
    m = 1.0 if not mul else c["mul"].double().abs()
    # the sum's error through act, act's own evaluation, the last sum's and rounding
    ey = (R.LIPSCHITZ[act] * ez + SUM32 * a) * m + _round_tol(ref, ref.abs() + a * m, y)
    if c["res"] is not None:
        ey = ey + 2.0 ** -23 * c["res"].double().abs()
    _close(out[live, :N], ref[live], ey[live] if torch.is_tensor(ey) else ey, "y")
    if keep:
        _close(pre[live], z[live], (ez + 1e-37)[live], "z")
        assert (pre[dead] == 7.0).all()
    if res == y:  # onto the residual itself, and the same bits
        both = args["residual"].clone()
        cep.cep_linear(desc, xb, c["w"], both, ws, **{**args, "residual": both})
        assert torch.equal(both[live, :N], out[live, :N])


GRADS = [
    # act, bias, mul, dy, dx, dw, add, pad
    (cep.CEP_IDENTITY, False, False, BF16, BF16, BF16, False, 0),
    (cep.CEP_IDENTITY, True, False, BF16, F32, F32, True, 8),
    (cep.CEP_IDENTITY, True, True, F32, BF16, F32, True, 0),
    (cep.CEP_RELU, True, True, F32, F32, BF16, False, 8),
    (cep.CEP_SILU, False, True, BF16, BF16, BF16, True, 0),
    (cep.CEP_GELU, True, False, F32, BF16, BF16, False, 16),
    (cep.CEP_GELU_TANH, True, True, BF16, F32, F32, True, 0),
]


@pytest.mark.parametrize("rows,d,N,groups", LINEARS)
@pytest.mark.parametrize("act,bias,mul,y,dxt,dwt,add,pad", GRADS)
def test_linear_backward(rows, d, N, groups, act, bias, mul, y, dxt, dwt, add, pad):
    c, off, dev, live, dead = _linear_case(rows, d, N, groups, act, bias, mul, None, pad,
                                           rows + d + N + 1)
    desc = _desc(rows, d, N, groups, act, None, y, pad, dx_dtype=dxt, dw_dtype=dwt)
    z = R.linear(c["x"], c["w"], c["bias"], None, None, 0, off)[0]
    pre = z.float()
    pre[dead] = NAN
    dy = c["dy"].to(DT[y])
    ref = R.linear_grad(torch.where(dead[:, None], 0.0, dy), c["x"], c["w"], pre.nan_to_num(0.0),
                        torch.where(dead[:, None], 0.0, c["mul"]) if mul else None, act, off)
    a = _randn(_gen(1), rows, d, dtype=DT[dxt]) if add else None
    out = dict(dx=torch.full((rows, d + 2 * pad), 7.0, dtype=DT[dxt], device="cuda"),
               dw=torch.full(c["w"].shape, 7.0, dtype=DT[dwt], device="cuda"),
               dbias=torch.full_like(c["bias"], 7.0) if bias else None,
               dmul=torch.full((rows, N + 2 * pad), 7.0, dtype=torch.bfloat16, device="cuda")
               if mul else None)
    args = dict(preact=pre, mul=_padded(c["mul"], N + 2 * pad) if mul else None, offsets=dev)
    ins = (_padded(dy, N + pad), _padded(c["x"], d + pad), c["w"],
           _space(cep.cep_linear_workspace(desc, True)))
    cep.cep_linear_backward(desc, *ins, dx_add=_padded(a, d + 2 * pad) if add else None, **args,
                            **out)
    up = dy.double().abs() * (c["mul"].double().abs() if mul else 1.0)
    # dz: the slope's evaluation, then its rounding
    e32 = 2.0 ** -16 * (1 + z.abs()) * up if act else SUM32 * up
    edz = torch.where(dead[:, None], 0.0, e32 + (1.02 * U16 + SUM32) * ref["dz"].abs())
    e32 = torch.where(dead[:, None], 0.0, e32 + SUM32 * ref["dz"].abs())
    dz0 = torch.zeros_like(z)  # tolerances: the same sums of magnitudes
    lim = R.linear_grad(edz, c["x"].nan_to_num(0.0).abs(), c["w"].abs(), dz0, None, 0, off)
    lim32 = R.linear_grad(e32, c["x"].nan_to_num(0.0).abs(), c["w"].abs(), dz0, None, 0, off)
    rdx = ref["dx"] if a is None else ref["dx"] + a.double()
    edx = lim["dx"] + _round_tol(rdx, rdx.abs() + (0 if a is None else a.double().abs()), dxt)
    _close(out["dx"][live, :d], rdx[live], edx[live], "dx")
    assert (out["dx"][dead] == 7.0).all() and (out["dx"][:, d:] == 7.0).all()
    _close(out["dw"], ref["dw"], lim["dw"] + _round_tol(ref["dw"], ref["dw"].abs(), dwt), "dw")
    if bias:
        _close(out["dbias"], ref["db"], lim32["db"] + 1e-37, "db")
    if mul:
        edm = 2.0 ** -16 * (1 + z.abs()) * dy.double().abs() + _round_tol(ref["dm"], ref["dm"].abs(), BF16)
        _close(out["dmul"][live, :N], ref["dm"][live], edm[live], "dmul")
        assert (out["dmul"][dead] == 7.0).all() and (out["dmul"][:, N:] == 7.0).all()
    # each output alone, dx onto dx_add
    for name, t in out.items():
        if t is None:
            continue
        alone = torch.full_like(t, 3.0)
        kw = dict(args)
        if name == "dx" and add:
            alone = _padded(a, d + 2 * pad)
            kw["dx_add"] = alone
        cep.cep_linear_backward(desc, *ins, **kw, **{name: alone})
        if name == "dx":  # its sums may be shared out differently then
            _close(alone[live, :d], rdx[live], edx[live], "dx alone")
        elif name == "dw":
            _close(alone, ref["dw"], lim["dw"] + _round_tol(ref["dw"], ref["dw"].abs(), dwt), "dw alone")
        elif name == "dmul":
            assert torch.equal(alone[live, :N], t[live, :N])
        else:
            assert torch.equal(alone, t)


LARGE = [
    # 256-wide tiles, the last of them in quarters
    (8700, 2056, 2056, 0), (8000, 2056, 2056, [2600, 20, 0, 2300, 1200, 1850]),
    # gradients: long tiles of more groups than are ordered by size, then of fewer
    (71685, 1032, 1032, [1024] * 70), (9000, 2056, 1544, [400, 5000, 70, 0, 3500]),
    # many short tiles of dW, and dx's before and behind them in one launch
    (2000, 1544, 1032, [60] * 31 + [100]), (4096, 520, 4104, [1500, 2500]),
    (5000, 4104, 520, [3000, 2000]),
]


@pytest.mark.parametrize("rows,d,N,groups", LARGE)
@pytest.mark.parametrize("case", range(6))
def test_linear_of_many_tiles(rows, d, N, groups, case):
    test_linear(rows, d, N, groups, *EXTRAS[case])


@pytest.mark.parametrize("rows,d,N,groups", LARGE)
@pytest.mark.parametrize("case", [0, 1, 3, 4, 6])
def test_linear_backward_of_many_tiles(rows, d, N, groups, case):
    test_linear_backward(rows, d, N, groups, *GRADS[case])


def test_linear_of_no_rows_has_zero_weight_gradients():
    for groups in (0, 3):
        desc = cep.make_linear(rows=0, d_in=64, d_out=32, n_groups=groups)
        off = torch.zeros(groups + 1, dtype=torch.int32, device="cuda") if groups else None
        dw = torch.full((max(groups, 1), 64, 32), 7.0, device="cuda")
        db = torch.full((max(groups, 1), 32), 7.0, device="cuda")
        cep.cep_linear_backward(desc, None, None, None,
                                _space(cep.cep_linear_workspace(desc, True)), dw=dw, dbias=db,
                                offsets=off)
        assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("T", [12, 33, 300])
@pytest.mark.parametrize("groups", [0, 3])
def test_linear_rows_do_not_affect_each_other(T, groups):
    # a NaN row, an infinite row and a zero row among ordinary ones
    d, N = 264, 136
    g = _gen(T)
    x, w = _randn(g, T, d), _randn(g, *[groups] * (groups > 0), d, N, std=0.05)
    off = torch.tensor([0, 5, 9, T], dtype=torch.int32, device="cuda") if groups else None
    desc = cep.make_linear(rows=T, d_in=d, d_out=N, n_groups=groups, y_dtype=BF16)
    ws = _space(cep.cep_linear_workspace(desc))
    y, x2 = torch.empty(T, N, dtype=torch.bfloat16, device="cuda"), x.clone()
    y2 = torch.empty_like(y)
    x2[3], x2[7, 7], x2[T - 1] = NAN, float("inf"), 0.0
    cep.cep_linear(desc, x, w, y, ws, offsets=off)
    cep.cep_linear(desc, x2, w, y2, ws, offsets=off)
    same = torch.ones(T, dtype=torch.bool, device="cuda")
    same[[3, 7, T - 1]] = False
    assert torch.equal(y[same], y2[same])
    assert torch.isnan(y2[3]).all() and (y2[T - 1] == 0).all() and not torch.isfinite(y2[7]).any()


@pytest.mark.parametrize("act", range(1, 5))
def test_linear_of_large_arguments(act):
    """Far from zero an activation is its argument or nothing, and its slope 1 or 0."""
    d = 8
    x = torch.zeros(4, d, device="cuda", dtype=torch.bfloat16)
    x[0, 0], x[1, 0], x[2, 0], x[3, 0] = 200.0, -200.0, 1e30, -1e30
    w = torch.zeros(d, d, device="cuda", dtype=torch.bfloat16)
    w[0] = 1.0
    desc = cep.make_linear(rows=4, d_in=d, d_out=d, act=act)
    ws = _space(cep.cep_linear_workspace(desc, True))
    y, pre, dx = (torch.empty(4, d, device="cuda") for _ in range(3))
    cep.cep_linear(desc, x, w, y, ws, preact=pre)
    want = x[:, :1].float().clamp_min(0)
    assert ((y - want).abs() <= 1e-30 + 2.0 ** -22 * want).all()
    cep.cep_linear_backward(desc, torch.ones_like(y), x, torch.eye(d, device="cuda").bfloat16(), ws,
                            dx=dx, preact=pre)
    assert torch.equal(dx, (want > 0).float().expand(4, d))


@pytest.mark.parametrize("rows", [1, 300])
def test_linear_gelu_and_its_slope_keep_their_digits(rows):
    """z on a grid over -14..14, as the bias of no product.  Half units in the last place of
    float32 (u): the fit of the distribution 2.9; 1 / (1 + 0.31 x) 3, which count 1.3 fold;
    the polynomial's steps one each, 8; the exponential 2 and its remainder's factor 2; the
    products 3: below 22 u of Phi(z) or the value, for which 32 u = 2^-19 is taken.  The
    density is within 6 u.  Below -12.9 Phi is subnormal, and what is lost there is less
    than 2^-122."""
    N, act = 16384, cep.CEP_GELU
    z = torch.linspace(-14, 14, N, device="cuda")
    d = 8
    x, w = torch.zeros(rows, d, device="cuda").bfloat16(), torch.zeros(d, N, device="cuda").bfloat16()
    desc = cep.make_linear(rows=rows, d_in=d, d_out=N, act=act)
    ws = _space(cep.cep_linear_workspace(desc, True))
    y, pre = torch.empty(rows, N, device="cuda"), torch.empty(rows, N, device="cuda")
    cep.cep_linear(desc, x, w, y, ws, bias=z, preact=pre)
    assert torch.equal(pre, z.expand(rows, N))
    zd = z.double()
    # (torch's ndtr is 1 + erf, which has 2 % of its value wrong at -8 and nothing left at -10)
    phi = torch.special.erfc(-zd / 2 ** 0.5) / 2
    value, slope = zd * phi, phi + zd * torch.exp(-zd * zd / 2) / (2 * torch.pi) ** 0.5
    far = torch.where(z < -12.9, 2.0 ** -122, 0.0)
    _close(y, value.expand(rows, N), 2.0 ** -19 * value.abs() + far, "y")
    # dbias: the slopes of a column, summed over one row of ones, the others zeros
    dy, db = torch.zeros(rows, N, device="cuda"), torch.empty(N, device="cuda")
    dy[rows // 2] = 1.0
    cep.cep_linear_backward(desc, dy, x, w, ws, dbias=db, preact=pre)
    _close(db, slope, 2.0 ** -19 * (phi + (slope - phi).abs()) + far, "slope")


@pytest.mark.parametrize("act", range(5))
def test_linear_gradient_of_a_row_that_is_no_number(act):
    """Its gradients, and the weights' where it counts, are none either."""
    T, d, N = 40, 64, 72
    g = _gen(act)
    x, w, mul = _randn(g, T, d), _randn(g, d, N, std=0.1), _randn(g, T, N)
    x[5] = NAN
    desc = cep.make_linear(rows=T, d_in=d, d_out=N, act=act)
    ws = _space(cep.cep_linear_workspace(desc, True))
    y, pre, dx = (torch.empty(T, n, device="cuda") for n in (N, N, d))
    dw, dm = torch.empty(d, N, device="cuda"), torch.empty_like(mul)
    cep.cep_linear(desc, x, w, y, ws, preact=pre, mul=mul)
    cep.cep_linear_backward(desc, torch.ones_like(y), x, w, ws, dx=dx, dw=dw, preact=pre, mul=mul,
                            dmul=dm)
    assert torch.isnan(y[5]).all() and torch.isnan(dm[5]).all() and torch.isnan(dw).all()
    assert act == 0 or torch.isnan(dx[5]).all()  # without an activation it hangs on dy alone
    for t in (y, dx, dm):
        assert torch.isfinite(t[torch.arange(T, device="cuda") != 5]).all()


@pytest.mark.parametrize("off", [[9, 5, 1, 0], [-7, 20, 1 << 30, -(1 << 30)], [0, 40, 0, 40],
                                 [50, 60, 70, 80], [0, 0, 0, 1 << 31 - 1]])
def test_linear_with_broken_offsets_stays_inside_its_arrays(off):
    """Rows hold anything then; what lies around the arrays is not touched."""
    rows, d, N = 40, 72, 136
    g = _gen(0)
    n = 3
    off = torch.tensor([v if v < 1 << 31 else v - (1 << 32) for v in off], dtype=torch.int32,
                       device="cuda")
    mk = lambda r, c, t=torch.bfloat16: torch.full((r + 400, c), 7.0, dtype=t, device="cuda")
    y, dx, dm, pre = mk(rows, N), mk(rows, d), mk(rows, N), mk(rows, N, torch.float32)
    x, w, mul, dy = _randn(g, rows, d), _randn(g, n, d, N), _randn(g, rows, N), _randn(g, rows, N)
    dw, db = torch.empty(n, d, N, device="cuda"), torch.empty(n, N, device="cuda")
    desc = cep.make_linear(rows=rows, d_in=d, d_out=N, n_groups=n, act=cep.CEP_SILU, y_dtype=BF16,
                           dx_dtype=BF16)
    need = cep.cep_linear_workspace(desc, True)
    ws = _space(need + 4096, 7)
    h = slice(200, 200 + rows)
    cep.cep_linear(desc, x, w, y[h], ws[:need], mul=mul, offsets=off, preact=pre[h])
    cep.cep_linear_backward(desc, dy, x, w, ws[:need], dx=dx[h], dw=dw, dbias=db, preact=pre[h],
                            mul=mul, dmul=dm[h], offsets=off)
    torch.cuda.synchronize()
    for t in (y, dx, dm, pre):
        assert (t[:200] == 7.0).all() and (t[200 + rows:] == 7.0).all()
    assert (ws[need:] == 7).all()


LOW, HIGH = -(1 << 31), (1 << 31) - 1  # of an offset
BROKEN = {
    "last lowest": lambda n, R: [*range(0, n)] + [LOW],
    "last near the lowest": lambda n, R: [0] + [R] * (n - 1) + [LOW + R // 2],
    "first lowest": lambda n, R: [LOW] + [R // n * i for i in range(1, n + 1)],
    "all highest": lambda n, R: [HIGH] * (n + 1),
    "last highest": lambda n, R: [0] * n + [HIGH],
    "ends apart": lambda n, R: [HIGH] + [R // 2] * (n - 1) + [LOW],
    "all rows in every second group": lambda n, R: [i % 2 * R for i in range(n + 1)],
    "descending": lambda n, R: [R - R // n * i for i in range(n + 1)],
    "between the ends": lambda n, R: [(LOW, HIGH, R // 2, -1, R)[i * i % 5] for i in range(n + 1)],
}


@pytest.mark.parametrize("rows,d,N,n", [
    (40, 72, 136, 3), (7, 72, 136, 3),          # streamed; one block of dz
    (130, 264, 136, 130),                       # streamed, more than 64 groups
    (900, 520, 264, 6), (2500, 264, 1032, 70),  # 128-wide tiles
    (8000, 2056, 2056, 6),                      # 256-wide ones, the last in quarters
    (4096, 520, 4104, 2), (9000, 2056, 1544, 5)])  # dx and dW in one launch
@pytest.mark.parametrize("kind", BROKEN)
def test_linear_with_offsets_of_any_number_stays_inside_its_arrays(rows, d, N, n, kind):
    off = BROKEN[kind](n, rows)
    assert len(off) == n + 1 and min(off) >= LOW and max(off) <= HIGH
    off = torch.tensor(off, dtype=torch.int32, device="cuda")
    g = _gen(1)
    guarded = {}

    def mk(name, *shape, dtype=torch.bfloat16):  # with 64 KB before and behind it
        size, pad = int(np.prod(shape)), 65536 // dtype.itemsize
        buf = guarded[name] = torch.full((size + 2 * pad,), 7, dtype=dtype, device="cuda")
        return buf[pad:pad + size].view(shape)

    y, pre = mk("y", rows, N), mk("preact", rows, N, dtype=torch.float32)
    dx, dm = mk("dx", rows, d), mk("dmul", rows, N)
    dw, db = mk("dw", n, d, N), mk("dbias", n, N, dtype=torch.float32)
    x, w, mul, dy = _randn(g, rows, d), _randn(g, n, d, N), _randn(g, rows, N), _randn(g, rows, N)
    desc = cep.make_linear(rows=rows, d_in=d, d_out=N, n_groups=n, act=cep.CEP_SILU, y_dtype=BF16,
                           dx_dtype=BF16, dw_dtype=BF16)
    ws = mk("workspace", cep.cep_linear_workspace(desc, True), dtype=torch.uint8)
    cep.cep_linear(desc, x, w, y, ws, mul=mul, offsets=off, preact=pre)
    out = dict(dx=dx, dw=dw, dbias=db, dmul=dm)
    cep.cep_linear_backward(desc, dy, x, w, ws, preact=pre, mul=mul, offsets=off, **out)
    for name, t in out.items():  # and each alone
        cep.cep_linear_backward(desc, dy, x, w, ws, preact=pre, mul=mul, offsets=off, **{name: t})
    torch.cuda.synchronize()
    for name, buf in guarded.items():
        pad = 65536 // buf.element_size()
        assert (buf[:pad] == 7).all() and (buf[-pad:] == 7).all(), name


# ------------------------------------------------------------ gate gradient

@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 256, 8), (5, 64, 8), (9, 7, 7), (70, 160, 8),
                                   (33, 129, 16), (130, 300, 3), (3, 1024, 16), (2000, 96, 6)])
@pytest.mark.parametrize("score,normalize,dtype,pad", [
    ("softmax", True, F32, 0), ("softmax", False, F32, 3), ("sigmoid", True, BF16, 1),
    ("sigmoid", False, F32, 0), ("softmax", False, BF16, 0)])
def test_gate_gradient(T, E, k, score, normalize, dtype, pad):
    g = _gen(T + E + k)
    l = _randn(g, T, E, dtype=DT[dtype], std=2.0)
    if T > 4 and E > 4:
        l[1, 2:] = float("-inf")  # fewer experts than slots
        l[2] = float("-inf")      # none
        l[3, ::2] = NAN           # masked too
        l[4, 1] = float("inf")
    kw = dict(score=score, normalize=normalize, scale=1.7)
    ids, _ = B.gate(l.float().cpu().numpy(), k, **kw)
    dw = _randn(g, T, k, dtype=torch.float32)
    dw[torch.from_numpy(ids < 0).cuda()] = NAN  # not used
    ids = torch.from_numpy(ids).cuda()
    if T > 4 and k > 2:
        ids[0, 1] = -7            # any id outside is an empty slot
        ids[0, 2] = E
        if T > 5:
            ids[5, 1] = ids[5, 0]  # the same expert twice
    desc = cep.make_gate(rows=T, n_experts=E, top_k=k, logit_dtype=dtype, normalize=normalize,
                         score=cep.CEP_SIGMOID if score == "sigmoid" else cep.CEP_SOFTMAX,
                         scale=1.7, ld=E + pad)
    out = torch.full((T, E + pad), 7.0, dtype=DT[dtype], device="cuda")
    cep.cep_gate_topk_backward(desc, _padded(l, E + pad), ids, dw, out)
    dwn = dw.nan_to_num(0.0).cpu().numpy()
    ref = R.gate_grad(l.float().cpu().numpy(), ids.cpu().numpy(), dwn, **kw)
    assert (out[:, E:] == 7.0).all()
    # a few float32 roundings of coefficients up to 1 times sums of |dw|, plus the
    # exponential's; the type's own rounding
    mag = torch.from_numpy(1.7 * np.abs(dwn).sum(1, keepdims=True)).cuda()
    ref = torch.from_numpy(ref).cuda()
    tol = 2.0 ** -18 * mag + (1.01 * U16 * ref.abs() if dtype == BF16 else 0)
    _close(out[:, :E], ref, tol, "d_logits")
    away = torch.ones(T, E, dtype=torch.bool, device="cuda")
    if score == "sigmoid" or normalize:  # experts that were not chosen: exactly nothing
        some = (ids >= 0) & (ids < E)
        t = some.nonzero()[:, 0]
        away[t, ids[some].long()] = False
    else:
        away = torch.isnan(l) | (l == float("-inf"))
    assert (out[:, :E][away] == 0).all()


def test_gate_gradient_of_far_scores():
    """Sigmoid scores near 0 and 1 keep the digits of 1 - s."""
    l = torch.tensor([[-80.0, -81.0, 30.0, 40.0, -100.0, 0.0]], device="cuda")
    ids = torch.tensor([[0, 1, 2, 3, 4, 5]], dtype=torch.int32, device="cuda")
    dw = torch.ones(1, 6, device="cuda")
    desc = cep.make_gate(rows=1, n_experts=6, top_k=6, score=cep.CEP_SIGMOID, scale=1.0)
    out = torch.empty_like(l)
    cep.cep_gate_topk_backward(desc, l, ids, dw, out)
    x = l.double()
    want = torch.sigmoid(x) * torch.sigmoid(-x)
    # subnormal scores have steps of 2^-149
    assert ((out - want).abs() <= 2.0 ** -20 * want + 2.0 ** -149).all()


# ----------------------------------------------- arrays past 2^31 elements

def test_sort_and_way_back_past_32_bits():
    T, k, d = 36000, 8, 8192  # 2.4e9 sorted values
    g = _gen(4)
    ids = torch.randint(-1, 12, (T, k), device="cuda", generator=g).int()
    x = _randn(g, T, d)
    sd = cep.make_expert_sort(rows=T, top_k=k, n_experts=12, capacity=T * k, row_bytes=2 * d)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    plan, pair, place = i32(14), i32(T * k), i32(T, k)
    xs = torch.empty(T * k, d, dtype=torch.bfloat16, device="cuda")
    cep.cep_expert_sort(sd, ids, plan, pair, place, _space(cep.cep_expert_sort_workspace(sd)), x=x,
                        out_x=xs)
    n = int(plan[12])
    assert n * d > 1 << 31
    for at in range(0, n, 20000):
        some = slice(at, min(at + 20000, n))
        assert torch.equal(xs[some], x[pair[some].long() // k])
    ud = cep.make_expert_unsort(rows=T, top_k=k, d=d, sorted_rows=n, ys_dtype=BF16, y_dtype=F32)
    y = torch.empty(T, d, device="cuda")
    cep.cep_expert_unsort(ud, xs, place, y)
    count = (place >= 0).sum(1, keepdim=True)
    # a token's own row, as often as it has experts: up to eight equal bf16 values, exact
    assert torch.equal(y, x.float() * count)
    dw = torch.empty(T, k, device="cuda")
    cep.cep_expert_unsort_backward(ud, y, xs, place, None, xs, dw)
    last = slice(n - 1000, n)
    want = y[pair[last].long() // k]
    _close(xs[last], want.double(), U16 * 1.01 * want.double().abs(), "dys")
    ref = (y[-500:].double() * x[-500:].double()).sum(1, keepdim=True)
    mag = (y[-500:].double() * x[-500:].double()).abs().sum(1, keepdim=True)
    _close(dw[-500:], torch.where(place[-500:] >= 0, ref, 0.0), SUM32 * mag.expand(-1, k), "dw")


@pytest.mark.parametrize("grouped", [False, True])
def test_linear_past_32_bits(grouped):
    rows, d, N = (1 << 20) + 77, 64, 2056  # 2.2e9 outputs
    g = _gen(6)
    off = [0, 5, (1 << 19) + 3, rows - 2] if grouped else None
    lead = (3,) if grouped else ()
    x, w = _randn(g, rows, d), _randn(g, *lead, d, N, std=0.1)
    dev = None if off is None else torch.tensor(off, dtype=torch.int32, device="cuda")
    desc = cep.make_linear(rows=rows, d_in=d, d_out=N, n_groups=3 if grouped else 0,
                           act=cep.CEP_SILU, y_dtype=BF16, dx_dtype=F32)
    ws = torch.empty(cep.cep_linear_workspace(desc, True), dtype=torch.uint8, device="cuda")
    y = torch.full((rows, N), 7.0, dtype=torch.bfloat16, device="cuda")
    pre, dx = torch.empty(rows, N, device="cuda"), torch.full((rows, d), 7.0, device="cuda")
    cep.cep_linear(desc, x, w, y, ws, offsets=dev, preact=pre)
    cep.cep_linear_backward(desc, y, x, w, ws, dx=dx, preact=pre, offsets=dev)  # dy: y itself
    for r, e in ((slice(0, 5), 0), (slice(5, 2000), 1), (slice(rows - 3000, rows - 2), 2)):
        we = w[e] if grouped else w
        z, ref, mag = R.linear(x[r], we, None, None, None, cep.CEP_SILU, None)
        _close(y[r], ref, 1.1 * SUM32 * mag + SUM32 * ref.abs() + U16 * 1.01 * ref.abs() + 1e-37, "y")
        grad = R.linear_grad(y[r], x[r], we, pre[r], None, cep.CEP_SILU, None)
        edz = 2.0 ** -16 * (1 + z.abs()) * y[r].double().abs() + (1.02 * U16 + SUM32) * grad["dz"].abs()
        _close(dx[r], grad["dx"], edz @ we.double().abs().T.contiguous() + 1e-37, "dx")
    if grouped:
        assert (y[-2:] == 7.0).all() and (dx[-2:] == 7.0).all()


# --------------------------------------------------------------- together

def test_replay_in_a_graph_beside_eager_work():
    """Sort, the products and the way back with every gradient, captured on one
    stream, with other inputs and eager calls (workspaces of their own) between the
    replays."""
    T, d, I, E, k = 700, 256, 136, 16, 4
    g = _gen(3)
    P = T * k
    logits, x, res = _randn(g, T, E, dtype=torch.float32), _randn(g, T, d), _randn(g, T, d)
    wg, wu = _randn(g, E, d, I, std=0.06), _randn(g, E, d, I, std=0.06)
    wd, bias = _randn(g, E, I, d, std=0.06), _randn(g, E, I, dtype=torch.float32)
    dout = _randn(g, T, d)
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device="cuda")
    f32, i32 = torch.float32, torch.int32
    gd = cep.make_gate(rows=T, n_experts=E, top_k=k, normalize=1, scale=1.0)
    sd = cep.make_expert_sort(rows=T, top_k=k, n_experts=E, capacity=P, row_bytes=2 * d)
    ud = cep.make_expert_unsort(rows=T, top_k=k, d=d, sorted_rows=P, ys_dtype=BF16, res_dtype=BF16,
                                y_dtype=BF16)
    up = cep.make_linear(rows=P, d_in=d, d_out=I, n_groups=E, y_dtype=BF16, dx_dtype=BF16,
                         dw_dtype=BF16)
    ga = cep.make_linear(rows=P, d_in=d, d_out=I, n_groups=E, act=cep.CEP_SILU, y_dtype=BF16,
                         dx_dtype=BF16, dw_dtype=BF16)
    dn = cep.make_linear(rows=P, d_in=I, d_out=d, n_groups=E, y_dtype=BF16, dx_dtype=BF16,
                         dw_dtype=BF16)

    def buffers():
        o = dict(ids=z(T, k, dt=i32), w=z(T, k, dt=f32), plan=z(E + 2, dt=i32), pair=z(P, dt=i32),
                 place=z(T, k, dt=i32), xs=z(P, d), u=z(P, I), h=z(P, I), pre=z(P, I, dt=f32),
                 ys=z(P, d), y=z(T, d), dys=z(P, d), dw=z(T, k, dt=f32), dl=z(T, E, dt=f32),
                 dh=z(P, I), du=z(P, I), dxs=z(P, d), dwd=z(E, I, d), dwg=z(E, d, I),
                 dwu=z(E, d, I), db=z(E, I, dt=f32), dx=z(T, d))
        ws = _space(max(cep.cep_expert_sort_workspace(sd),
                        *(cep.cep_linear_workspace(q, True) for q in (up, ga, dn))))
        return o, ws

    def step(o, ws, s):
        cep.cep_gate_topk(gd, logits, None, o["ids"], o["w"], stream=s)
        cep.cep_expert_sort(sd, o["ids"], o["plan"], o["pair"], o["place"], ws, x=x, out_x=o["xs"],
                            stream=s)
        n = dict(offsets=o["plan"], stream=s)
        cep.cep_linear(up, o["xs"], wu, o["u"], ws, **n)
        cep.cep_linear(ga, o["xs"], wg, o["h"], ws, bias=bias, mul=o["u"], preact=o["pre"], **n)
        cep.cep_linear(dn, o["h"], wd, o["ys"], ws, **n)
        cep.cep_expert_unsort(ud, o["ys"], o["place"], o["y"], w=o["w"], residual=res, stream=s)
        cep.cep_expert_unsort_backward(ud, dout, o["ys"], o["place"], o["w"], o["dys"], o["dw"],
                                       stream=s)
        cep.cep_gate_topk_backward(gd, logits, o["ids"], o["dw"], o["dl"], stream=s)
        cep.cep_linear_backward(dn, o["dys"], o["h"], wd, ws, dx=o["dh"], dw=o["dwd"], **n)
        cep.cep_linear_backward(ga, o["dh"], o["xs"], wg, ws, dx=o["dxs"], dw=o["dwg"],
                                dbias=o["db"], preact=o["pre"], mul=o["u"], dmul=o["du"], **n)
        cep.cep_linear_backward(up, o["du"], o["xs"], wu, ws, dx=o["dxs"], dw=o["dwu"],
                                dx_add=o["dxs"], **n)
        cep.cep_expert_unsort(ud, o["dxs"], o["place"], o["dx"], residual=dout, stream=s)

    captured, ws1 = buffers()
    eager, ws2 = buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured, ws1, torch.cuda.current_stream())
    for i in range(4):
        x.copy_(_randn(g, T, d))
        logits.copy_(_randn(g, T, E, dtype=f32, std=3.0))
        for t in (*eager.values(), *captured.values()):
            t.zero_()
        step(eager, ws2, None)
        graph.replay()
        step(eager, ws2, None)
        torch.cuda.synchronize()
        for name in eager:
            assert torch.equal(eager[name], captured[name]), (i, name)


def _whole_block(b, experts, x, res, k):
    """The block in float64 as a function that autograd differentiates, with the
    choice of experts held fixed; its leaves by name."""
    leaf = lambda t: t.detach().double().requires_grad_()
    p = dict(x=leaf(x), norm=leaf(b.norm), gate=leaf(b.gate),
             **{n: leaf(t) for n, t in zip(("wg", "wu", "wd"), experts)})
    s = p["x"] + res.double()
    y = s / torch.sqrt((s * s).mean(-1, keepdim=True) + 1e-6) * p["norm"]
    logits = y @ p["gate"]
    w = torch.softmax(logits.gather(1, b.ids[:len(x)].long()), -1)
    ffn = lambda a, wg, wu, wd: (torch.nn.functional.silu(a @ wg) * (a @ wu)) @ wd
    out = ffn(y, *(t.double() for t in b.shared))
    for e in range(len(experts[0])):
        coef = torch.where(b.ids[:len(x)] == e, w, 0.0).sum(1, keepdim=True)
        out = out + coef * ffn(y, p["wg"][e], p["wu"][e], p["wd"][e])
    return out, p


@pytest.mark.parametrize("T", [1, 9, 300])
def test_block_gradients_through_the_routed_experts(T):
    """MoEBlock and RoutedExperts together against the whole block differentiated in
    float64: sums of terms with at most four bf16 roundings of random signs each on
    their way (y, h, the gradients of z and of a sorted row): 2^-8 / 3^.5 each, and
    a margin of two.  The gate's gradient has no such averaging: a coefficient's is
    one product, <d_out, expert's row>, whose error is up to |d_out| times that of the
    row (Cauchy-Schwarz), and c_j (g_j - sum c g) at most doubles the largest."""
    from paper_2609_33252_amd import moe_block
    d, I, E, k = 256, 128, 8, 3
    g = _gen(T)
    n = lambda *s, std=0.08: _randn(g, *s, std=std)
    experts = [n(E, d, I), n(E, d, I), n(E, I, d)]
    b = moe_block.MoEBlock(d=d, d_ff=I, d_shared=200, n_experts=E, top_k=k, n_ranks=1, rank=0,
                           max_tokens=300, norm=1 + n(d).float(), gate=n(d, E).float(),
                           shared=(n(d, 200), n(d, 200), n(200, d)),
                           experts=cep.make_weights(*experts), w_dtype=cep.CEP_BF16)
    routed = moe_block.RoutedExperts(top_k=k, w_gate=experts[0], w_up=experts[1],
                                     w_down=experts[2])
    # the sum x + residual is exact in bf16: it is saved without a rounding of its own
    x = (torch.randint(-32, 33, (T, d), device="cuda", generator=g) / 16).bfloat16()
    res, dout = torch.zeros_like(x), n(T, d, std=1.0)
    out = b.forward(x, res, train=True)
    total = routed.forward(b.y[:T], b.ids[:T], b.w[:T], train=True)
    d_y, d_w, dw = routed.backward(dout)
    again = routed.backward(dout.float())
    d_gate_y, d_gate = b.gate_backward(d_w)
    dx, d_norm, _ = b.backward(dout, d_y=d_y + d_gate_y)
    ref, p = _whole_block(b, experts, x, torch.zeros_like(x), k)
    ref.backward(dout.double())
    lim = 2 * (4 / 3) ** 0.5 * 2.0 ** -8
    rel = lambda got, want: float((got.double() - want).norm() / want.norm().clamp_min(1e-30))
    assert rel(total + b.shared_y[:T], ref.detach()) < lim
    assert rel(out, ref.detach()) < lim
    place, rows = routed.saved[1], routed.saved[-1]
    worst = rows[place.long().flatten()].double().norm(dim=1).view(T, k).amax(1)
    most = (b.y[:T].double().norm(dim=1) * 2 * lim * worst * dout.double().norm(dim=1)).sum()
    want = p["gate"].grad
    assert (d_gate.double() - want).norm() < lim * want.norm() + most
    for name, got in (("x", dx), ("norm", d_norm), ("wg", dw[0]), ("wu", dw[1]), ("wd", dw[2])):
        assert rel(got, p[name].grad) < lim, name
    assert torch.equal(again[1], d_w) and all(torch.equal(a, c) for a, c in zip(again[2], dw))
    b.close()


def test_routed_experts_on_two_streams():
    """Two sets of experts at work at once, each on a stream of its own, the backward
    pass on another one than the forward pass."""
    from paper_2609_33252_amd import moe_block
    T, d, I, E, k = 500, 256, 264, 6, 3
    g = _gen(8)
    n = lambda *s: _randn(g, *s, std=0.1)
    sets = []
    for _ in range(2):
        r = moe_block.RoutedExperts(top_k=k, w_gate=n(E, d, I), w_up=n(E, d, I), w_down=n(E, I, d))
        ids = torch.randint(-1, E, (T, k), device="cuda", generator=g).int()
        sets.append((r, _randn(g, T, d), ids, torch.rand(T, k, device="cuda", generator=g), n(T, d)))

    def alone(r, y, ids, c, dt):
        out = r.forward(y, ids, c, train=True)
        return [out, *(lambda a, b, e: [a, b, *e])(*r.backward(dt))]

    want = [alone(*s) for s in sets]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for (r, y, ids, c, dt), s in zip(sets, streams):
            with torch.cuda.stream(s):
                got.append([r.forward(y, ids, c, train=True)])
        for s in streams[:2]:
            streams[2].wait_stream(s)
        for (r, *_, dt), o in zip(sets, got):
            with torch.cuda.stream(streams[2]):
                d_y, d_c, dw = r.backward(dt)
                o += [d_y, d_c, *dw]
        torch.cuda.synchronize()
        for w, o in zip(want, got):
            assert all(torch.equal(a, b) for a, b in zip(w, o))
    # torch hands out its 32 streams in turn, and the readiness tests depend on which
    # hardware queues theirs are on: the turn ends where it began
    for _ in range(32 - len(streams)):
        torch.cuda.Stream()


def test_routed_experts_refuse_what_their_operators_would_misread():
    from paper_2609_33252_amd import moe_block
    bf = dict(dtype=torch.bfloat16, device="cuda")
    w = [torch.zeros(4, 64, 32, **bf), torch.zeros(4, 64, 32, **bf), torch.zeros(4, 32, 64, **bf)]
    make = lambda a, b, c: moe_block.RoutedExperts(top_k=2, w_gate=a, w_up=b, w_down=c)
    for i in range(3):
        for wrong in (w[i].float(), w[i][:3], w[i].cpu(), w[i].transpose(1, 2)):
            with pytest.raises(ValueError):
                make(*[wrong if j == i else w[j] for j in range(3)])
    r = make(*w)
    y, ids = torch.zeros(8, 64, **bf), torch.zeros(8, 2, dtype=torch.int32, device="cuda")
    c = torch.ones(8, 2, device="cuda")
    with pytest.raises(ValueError):
        r.backward(y)
    for bad in ((y.float(), ids, c), (y[:, :32], ids, c), (y, ids.long(), c), (y, ids, c.double()),
                (y, ids[:7], c), (torch.zeros(9, 64, **bf), ids, c), (y.t(), ids, c)):
        with pytest.raises(ValueError):
            r.forward(*bad)
    r.forward(y, ids, c)
    with pytest.raises(ValueError):
        r.backward(y)  # that pass kept nothing
    r.forward(y, ids, c, train=True)
    with pytest.raises(ValueError):
        r.backward(y[:7])


def test_routed_experts_of_no_tokens():
    from paper_2609_33252_amd import moe_block
    bf = dict(dtype=torch.bfloat16, device="cuda")
    r = moe_block.RoutedExperts(top_k=2, w_gate=torch.ones(4, 64, 32, **bf),
                                w_up=torch.ones(4, 64, 32, **bf), w_down=torch.ones(4, 32, 64, **bf))
    for T in (0, 3):  # no tokens; tokens of no expert
        ids = torch.full((T, 2), -1, dtype=torch.int32, device="cuda")
        out = r.forward(torch.ones(T, 64, **bf), ids, torch.ones(T, 2, device="cuda"), train=True)
        d_y, d_w, dw = r.backward(torch.ones(T, 64, **bf))
        assert (out == 0).all() and (d_y == 0).all() and (d_w == 0).all()
        assert all((t == 0).all() for t in dw)


@pytest.mark.parametrize("seed", [0, 1])
def test_routed_experts_match_differences(seed):
    """Directional derivatives of the float64 form beside the gradients' product with
    the direction, at the same tolerance as against the formula."""
    from paper_2609_33252_amd import moe_block
    T, d, I, E, k = 40, 64, 40, 5, 2
    g = _gen(seed + 50)
    w = [_randn(g, E, d, I, std=0.2), _randn(g, E, d, I, std=0.2), _randn(g, E, I, d, std=0.2)]
    r = moe_block.RoutedExperts(top_k=k, w_gate=w[0], w_up=w[1], w_down=w[2])
    y, dt = _randn(g, T, d), _randn(g, T, d)
    ids = torch.randint(-1, E, (T, k), device="cuda", generator=g).int()
    c = torch.rand(T, k, device="cuda", generator=g)
    r.forward(y, ids, c, train=True)
    d_y, d_c, dw = r.backward(dt)

    def f(y, c, wg, wu, wd):
        out = torch.zeros(T, d, dtype=torch.float64, device="cuda")
        for e in range(E):
            coef = torch.where(ids == e, c, 0.0).sum(1, keepdim=True)
            out += coef * B.gated_ffn(y, wg[e], wu[e], wd[e])[3]
        return (out * dt.double()).sum()

    at = [t.double() for t in (y, c, *w)]
    for i, grad in enumerate((d_y, d_c, *dw)):
        # along the gradient itself: the product is its square's sum, and the bf16
        # roundings on the way (2^-8 each, four) carry over as they are
        v = grad.double() / grad.double().norm()
        h = 1e-4
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + h * v, at[i] - h * v
        slope = float(f(*up) - f(*down)) / (2 * h)
        assert abs(slope / float(grad.double().norm()) - 1) < 4 * U16, i


def _small_block(seed, T, d=256, I=128, E=8, k=3):
    """A block with its experts in both forms; inputs as of the block before."""
    from paper_2609_33252_amd import moe_block
    g = _gen(seed)
    n = lambda *s, std=0.08: _randn(g, *s, std=std)
    experts = [n(E, d, I), n(E, d, I), n(E, I, d)]
    b = moe_block.MoEBlock(d=d, d_ff=I, d_shared=200, n_experts=E, top_k=k, n_ranks=1, rank=0,
                           max_tokens=T, norm=1 + n(d).float(), gate=n(d, E).float(),
                           shared=(n(d, 200), n(d, 200), n(200, d)),
                           experts=cep.make_weights(*experts), w_dtype=cep.CEP_BF16)
    routed = moe_block.RoutedExperts(top_k=k, w_gate=experts[0], w_up=experts[1],
                                     w_down=experts[2])
    return g, b, routed, n(T, d, std=1.0), n(T, d, std=1.0)


def test_gate_gradient_is_of_the_pass_that_was_saved():
    """The buffers that a pass leaves its choice in may change before the backward pass."""
    T = 9
    g, b, _, x, res = _small_block(21, T)
    b.forward(x, res, train=True)
    d_w = _randn(g, T, 3, dtype=torch.float32)
    want = b.gate_backward(d_w)
    b.ids.copy_((b.ids + 1) % 8)
    got = b.gate_backward(d_w)
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    b.close()


@pytest.mark.parametrize("T", [1, 9, 300])
def test_gate_weight_gradient_from_given_coefficients(T):
    """MoEBlock.gate_backward alone: from the d_topk_w that it gets.  A logit's gradient is
    within 2^-18 of the row's sum of |d_topk_w| (as in test_gate_gradient), and the float32
    products within 2^-12 of the sum of magnitudes."""
    g, b, _, x, res = _small_block(T + 30, T)
    b.forward(x, res, train=True)
    d_w = _randn(g, T, 3, dtype=torch.float32)
    d_y, d_gate = b.gate_backward(d_w)
    y, logits = b.y[:T].double(), b.y[:T].float() @ b.gate
    dl = torch.from_numpy(R.gate_grad(logits.cpu().numpy(), b.ids[:T].cpu().numpy(),
                                      d_w.cpu().numpy(), normalize=True)).cuda()
    e = (2.0 ** -18 * d_w.double().abs().sum(1, keepdim=True)).expand_as(dl)
    across = lambda a, c: a.T.contiguous() @ c
    want, tol = across(y, dl), across(y.abs(), e + 2.0 ** -12 * dl.abs())
    assert tol.norm() < 2.0 ** -6 * want.norm()  # a check that can fail
    _close(d_gate, want, tol, "d_gate")
    gate = b.gate.double().T.contiguous()
    want, tol = dl @ gate, (e + 2.0 ** -12 * dl.abs()) @ gate.abs()
    assert tol.norm() < 2.0 ** -6 * want.norm()
    _close(d_y, want, tol, "d_y")
    b.close()


@pytest.mark.parametrize("T", [1, 9, 300])
def test_gate_weight_gradient_through_the_routed_experts(T):
    """From d_out through the experts' rows to the gate's weight, against float64 from the
    block's own y on.  A coefficient's gradient is <d_out, row>; on the way to the row u, h
    and the row itself are rounded to bf16, each by a part of at most 2^-8 / 3^.5 (r.m.s.)
    with a sign of its own, so that its variance is the sum of the squares of those parts
    times the derivatives.  Six deviations, of variances carried on through the choice's
    Jacobian and the product with y, are taken for a gradient."""
    d, I, E, k = 256, 128, 8, 3
    g, b, routed, x, res = _small_block(T + 40, T)
    b.forward(x, res, train=True)
    y, ids, w = b.y[:T], b.ids[:T], b.w[:T]
    dout = _randn(g, T, d)
    routed.forward(y, ids, w, train=True)
    d_w = routed.backward(dout)[1]
    d_gate = b.gate_backward(d_w)[1]
    part = 2.0 ** -8 / 3 ** 0.5
    yd, dd = y.double(), dout.double()
    rows, var = (torch.empty(T, k, dtype=torch.float64, device="cuda") for _ in range(2))
    for t in range(T):
        for j, e in enumerate(ids[t].tolist()):
            z, u = (yd[t] @ m[e].double() for m in (routed.w_gate, routed.w_up))
            h, wd = z * torch.sigmoid(z) * u, routed.w_down[e].double()
            row = h @ wd
            rows[t, j] = (dd[t] * row).sum()
            var[t, j] = part ** 2 * ((dd[t] * row).square().sum()
                                     + 2 * ((wd @ dd[t]) * h).square().sum())
    _close(d_w, rows, 6 * var.sqrt() + SUM32 * rows.abs(), "d_w")
    logits = yd @ b.gate.double()
    c = torch.softmax(logits.gather(1, ids.long()), 1)
    jac = torch.diag_embed(c) - c[:, :, None] * c[:, None, :]
    to_experts = lambda v: torch.zeros(T, E, dtype=torch.float64, device="cuda").scatter(
        1, ids.long(), v)
    dl = to_experts((jac * rows[:, None, :]).sum(2))
    vl = to_experts((jac.square() * var[:, None, :]).sum(2))
    across = lambda a, c: a.T.contiguous() @ c
    want = across(yd, dl)
    tol = 6 * across(yd.square(), vl).sqrt() + 2.0 ** -12 * across(yd.abs(), dl.abs())
    assert tol.norm() < 2.0 ** -4 * want.norm()  # a check that can fail
    _close(d_gate, want, tol, "d_gate")
    b.close()


def test_routed_experts_raise_for_ids_of_no_expert():
    from paper_2609_33252_amd import moe_block
    T, d, I, E, k = 40, 64, 40, 5, 2
    g = _gen(60)
    r = moe_block.RoutedExperts(top_k=k, w_gate=_randn(g, E, d, I), w_up=_randn(g, E, d, I),
                                w_down=_randn(g, E, I, d))
    y, c = _randn(g, T, d), torch.rand(T, k, device="cuda", generator=g)
    good = torch.randint(-1, E, (T, k), device="cuda", generator=g).int()
    want = r.forward(y, good, c, train=True)
    assert int(r.bad_ids) == 0 and r.saved is not None
    for wrong in (E, -2, 2 ** 31 - 1, -2 ** 31):
        ids = good.clone()
        ids[3, 1] = ids[7, 0] = wrong
        with pytest.raises(RuntimeError, match="2 expert ids"):
            r.forward(y, ids, c, train=True)
        assert int(r.bad_ids) == 2
        with pytest.raises(ValueError):
            r.backward(want)  # that pass kept nothing
    # captured: the slots are empty, and counted
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = r.forward(y, ids, c)
    bad = r.bad_ids
    empty = torch.where(ids == wrong, -1, ids).int()
    want = r.forward(y, empty, c)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and int(bad) == 2
    ids.copy_(empty)
    graph.replay()
    assert torch.equal(out, want) and int(bad) == 0


def test_routed_experts_sum_the_gradient_of_y_in_float32():
    """Whole numbers that every rounding to bf16 of rows and products keeps: z is 64, where
    SiLU is its argument and its slope 1.  The gradient of y, a sum of sums beyond eight
    bits, has to be exact."""
    from paper_2609_33252_amd import moe_block
    T, d, I, E, k = 40, 16, 24, 4, 2
    g = _gen(61)
    whole = lambda lo, hi, *s: torch.randint(lo, hi + 1, s, device="cuda", generator=g).bfloat16()
    wg, wu, wd = whole(-7, 7, E, d, I), whole(-7, 7, E, d, I), whole(-1, 1, E, I, d)
    wg[:, 0], wu[:, 0] = 64, whole(1, 3, E, I)
    y = torch.zeros(T, d, device="cuda").bfloat16()
    y[:, 0] = 1
    ids = torch.rand(T, E, device="cuda", generator=g).topk(k, -1)[1].int()
    c = torch.tensor([1.0, 0.5], device="cuda").expand(T, k).contiguous()
    dt = 2 * whole(-2, 2, T, d)
    r = moe_block.RoutedExperts(top_k=k, w_gate=wg, w_up=wu, w_down=wd)
    r.forward(y, ids, c, train=True)
    d_y = r.backward(dt)[0]
    want = torch.zeros(T, d, dtype=torch.float64, device="cuda")
    parts = []
    for t in range(T):
        for j, e in enumerate(ids[t].tolist()):
            dh = wd[e].double() @ (c[t, j].double() * dt[t].double())
            dz, du = dh * wu[e, 0].double(), 64 * dh
            assert torch.equal(dz, dz.bfloat16().double()) and torch.equal(du, du.bfloat16().double())
            parts += [wg[e].double() @ dz, wu[e].double() @ du]
            want[t] += parts[-1] + parts[-2]
    parts = torch.stack(parts)
    assert not torch.equal(parts, parts.bfloat16().double()) and float(parts.abs().max()) < 2 ** 24
    assert torch.equal(d_y.double(), want)


def test_a_pass_that_fails_leaves_nothing_to_go_back_through(monkeypatch):
    T = 9
    g, b, routed, x, res = _small_block(70, T)
    b.forward(x, res, train=True)
    routed.forward(b.y[:T], b.ids[:T], b.w[:T], train=True)

    def fails(*a, **kw):
        raise cep.CepError(cep.CEP_ENOMEM, "cep")

    with monkeypatch.context() as m:
        m.setattr(cep, "cep_linear", fails)
        m.setattr(cep, "cep_dispatch", fails)
        with pytest.raises(cep.CepError):
            routed.forward(b.y[:T], b.ids[:T], b.w[:T], train=True)
        with pytest.raises(cep.CepError):
            b.forward(x, res, train=True)
    with pytest.raises(ValueError):
        routed.backward(x)
    with pytest.raises(ValueError):
        b.backward(x)
    with pytest.raises(ValueError):
        b.gate_backward(torch.zeros(T, 3, device="cuda"))
    b.forward(x, res, train=True)
    assert len(b.backward(x)) == 3
    b.close()
