"""The operators that train through the routed experts without a GPU: refusals
come before any HIP call, and the formulas that the GPU tests compare with agree
with differences."""
import ctypes
import os

import numpy as np
import pytest
import torch

from paper_2609_33252_amd import cep

from . import _block_ref as B
from . import _train_ref as R

PTR = 1 << 20  # an aligned address that no refused call reads
BIG = torch.empty(1 << 24, dtype=torch.uint8)


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(cep.LIB_PATH):
        from paper_2609_33252_amd import build
        build.build()


def _refused(status, fn, *a, **kw):
    with pytest.raises(cep.CepError) as e:
        fn(*a, **kw)
    assert e.value.status == status
    assert fn.__name__ in str(e.value)


def test_descriptors_match_the_header():
    # the sizes a C compiler gives the header's structs
    assert ctypes.sizeof(cep.cep_expert_sort_desc) == 32
    assert ctypes.sizeof(cep.cep_expert_unsort_desc) == 56
    assert ctypes.sizeof(cep.cep_linear_desc) == 80


# ------------------------------------------------------------------- sort

def _sort(**kw):
    return cep.make_expert_sort(**{**dict(rows=4, top_k=2, n_experts=8, capacity=8, row_bytes=64),
                                   **kw})


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=(1 << 21) + 1), dict(top_k=0),
                                 dict(top_k=17), dict(n_experts=0), dict(n_experts=1025),
                                 dict(row_bytes=0), dict(row_bytes=131073), dict(ld_x=63),
                                 dict(ld_x=-64), dict(capacity=-1)])
def test_sort_refuses_descriptors(bad):
    _refused(cep.CEP_EINVAL, cep.cep_expert_sort, _sort(**bad), PTR, PTR, PTR, PTR, BIG, x=PTR,
             out_x=PTR)
    assert cep.cep_expert_sort_workspace(_sort(**bad)) == 0


def test_sort_refuses_arguments():
    f = cep.cep_expert_sort
    _refused(cep.CEP_EINVAL, f, None, PTR, PTR, PTR, PTR, BIG)
    _refused(cep.CEP_ENOMEM, f, _sort(capacity=7), PTR, PTR, PTR, PTR, BIG)
    for i in range(4):
        for wrong in (None, PTR + 2):
            _refused(cep.CEP_EINVAL, f, _sort(), *[wrong if j == i else PTR for j in range(4)], BIG)
    _refused(cep.CEP_EINVAL, f, _sort(), PTR, PTR, PTR, PTR, BIG, x=PTR)
    _refused(cep.CEP_EINVAL, f, _sort(), PTR, PTR, PTR, PTR, BIG, out_x=PTR)
    _refused(cep.CEP_EINVAL, f, _sort(), PTR, PTR, PTR, PTR, None)
    _refused(cep.CEP_ENOMEM, f, _sort(), PTR, PTR, PTR, PTR, BIG[:16])
    _refused(cep.CEP_EINVAL, f, _sort(rows=0), None, None, None, None, BIG)
    assert cep.cep_expert_sort_workspace(_sort(rows=1 << 21, top_k=16, n_experts=1024)) \
        == 4 * ((1 << 25) // 1024 + 1) * 1025


# ----------------------------------------------------------------- unsort

def _unsort(**kw):
    return cep.make_expert_unsort(**{**dict(rows=4, top_k=2, d=64, sorted_rows=8), **kw})


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=(1 << 21) + 1), dict(top_k=0),
                                 dict(top_k=17), dict(d=0), dict(d=32769), dict(sorted_rows=-1),
                                 dict(ys_dtype=2), dict(res_dtype=4), dict(y_dtype=-1),
                                 dict(ld_ys=63), dict(ld_res=1), dict(ld_y=-64)])
def test_unsort_refuses_descriptors(bad):
    _refused(cep.CEP_EINVAL, cep.cep_expert_unsort, _unsort(**bad), PTR, PTR, PTR)
    _refused(cep.CEP_EINVAL, cep.cep_expert_unsort_backward, _unsort(**bad), PTR, PTR, PTR, PTR,
             PTR, PTR)


def test_unsort_refuses_arguments():
    f, b = cep.cep_expert_unsort, cep.cep_expert_unsort_backward
    _refused(cep.CEP_EINVAL, f, None, PTR, PTR, PTR)
    _refused(cep.CEP_EINVAL, b, None, PTR, PTR, PTR, PTR, PTR, PTR)
    for i in range(3):
        for wrong in (None, PTR + 1):
            _refused(cep.CEP_EINVAL, f, _unsort(), *[wrong if j == i else PTR for j in range(3)])
    _refused(cep.CEP_EINVAL, f, _unsort(), PTR, PTR, PTR, w=PTR + 2)
    _refused(cep.CEP_EINVAL, f, _unsort(), PTR, PTR, PTR, residual=PTR + 2)
    for i in range(3):
        _refused(cep.CEP_EINVAL, b, _unsort(), *[None if j == i else PTR for j in range(3)], PTR,
                 PTR, PTR)
    for i in range(6):
        _refused(cep.CEP_EINVAL, b, _unsort(), *[PTR + 1 if j == i else PTR for j in range(6)])
    _refused(cep.CEP_EINVAL, b, _unsort(), PTR, PTR, PTR, PTR, None, None)
    f(_unsort(rows=0), None, None, None)  # nothing to do, nothing launched
    b(_unsort(rows=0), None, None, None, None, None, None)


# ----------------------------------------------------------------- linear

def _linear(**kw):
    return cep.make_linear(**{**dict(rows=4, d_in=64, d_out=32), **kw})


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=(1 << 21) + 1), dict(d_in=0),
                                 dict(d_in=12), dict(d_in=32776), dict(d_out=4), dict(d_out=-8),
                                 dict(n_groups=-1), dict(n_groups=1025), dict(act=-1), dict(act=5),
                                 dict(y_dtype=2), dict(res_dtype=3), dict(dx_dtype=4),
                                 dict(dw_dtype=-1), dict(ld_x=56), dict(ld_x=68), dict(ld_y=24),
                                 dict(ld_mul=36), dict(ld_res=-32), dict(ld_dx=32),
                                 dict(ld_x=(1 << 21) + 8)])
def test_linear_refuses_descriptors(bad):
    off = PTR if bad.get("n_groups") else None
    _refused(cep.CEP_EINVAL, cep.cep_linear, _linear(**bad), PTR, PTR, PTR, BIG, offsets=off)
    _refused(cep.CEP_EINVAL, cep.cep_linear_backward, _linear(**bad), PTR, PTR, PTR, BIG, dx=PTR,
             offsets=off)
    assert cep.cep_linear_workspace(_linear(**bad)) == 0
    assert cep.cep_linear_workspace(_linear(**bad), True) == 0


def test_linear_refuses_arguments():
    f, b = cep.cep_linear, cep.cep_linear_backward
    assert BIG.data_ptr() % 16 == 0
    _refused(cep.CEP_EINVAL, f, None, PTR, PTR, PTR, BIG)
    _refused(cep.CEP_EINVAL, b, None, PTR, PTR, PTR, BIG, dx=PTR)
    for i in range(3):
        for wrong in (None, PTR + 8):
            _refused(cep.CEP_EINVAL, f, _linear(), *[wrong if j == i else PTR for j in range(3)],
                     BIG)
    for name in ("bias", "mul", "residual", "preact"):
        _refused(cep.CEP_EINVAL, f, _linear(), PTR, PTR, PTR, BIG, **{name: PTR + 8})
    # offsets go with groups
    _refused(cep.CEP_EINVAL, f, _linear(), PTR, PTR, PTR, BIG, offsets=PTR)
    _refused(cep.CEP_EINVAL, f, _linear(n_groups=2), PTR, PTR, PTR, BIG)
    _refused(cep.CEP_EINVAL, f, _linear(n_groups=2), PTR, PTR, PTR, BIG, offsets=PTR + 2)
    _refused(cep.CEP_EINVAL, f, _linear(), PTR, PTR, PTR, None)
    _refused(cep.CEP_ENOMEM, f, _linear(), PTR, PTR, PTR, BIG[:64])
    out = dict(dx=PTR, dw=PTR)
    for i in range(3):
        _refused(cep.CEP_EINVAL, b, _linear(), *[None if j == i else PTR for j in range(3)], BIG,
                 **out)
        _refused(cep.CEP_EINVAL, b, _linear(), *[PTR + 8 if j == i else PTR for j in range(3)],
                 BIG, **out)
    for name in ("dx", "dw", "dbias", "preact", "mul", "dmul", "dx_add"):
        kw = {**out, "mul": PTR, "preact": PTR, name: PTR + 8}
        _refused(cep.CEP_EINVAL, b, _linear(), PTR, PTR, PTR, BIG, **kw)
    _refused(cep.CEP_EINVAL, b, _linear(), PTR, PTR, PTR, BIG)  # no output
    _refused(cep.CEP_EINVAL, b, _linear(act=cep.CEP_SILU), PTR, PTR, PTR, BIG, **out)  # no preact
    _refused(cep.CEP_EINVAL, b, _linear(), PTR, PTR, PTR, BIG, dw=PTR, dx_add=PTR)
    _refused(cep.CEP_EINVAL, b, _linear(), PTR, PTR, PTR, BIG, dx=PTR, dmul=PTR, preact=PTR)
    _refused(cep.CEP_EINVAL, b, _linear(), PTR, PTR, PTR, BIG, dx=PTR, dmul=PTR, mul=PTR)
    _refused(cep.CEP_EINVAL, b, _linear(n_groups=2), PTR, PTR, PTR, BIG, **out)
    _refused(cep.CEP_EINVAL, b, _linear(), PTR, PTR, PTR, None, **out)
    _refused(cep.CEP_ENOMEM, b, _linear(), PTR, PTR, PTR, BIG[:64], **out)
    f(_linear(rows=0), None, None, None, None)  # nothing to do, nothing launched


def test_linear_refuses_outputs_over_its_inputs():
    f, b = cep.cep_linear, cep.cep_linear_backward
    x, w, y = PTR, PTR + 1024, PTR + 2048
    _refused(cep.CEP_EINVAL, f, _linear(), x, w, x, BIG)
    _refused(cep.CEP_EINVAL, f, _linear(), x, w, y, BIG, preact=x)
    _refused(cep.CEP_EINVAL, f, _linear(), x, w, y, BIG, preact=y)
    _refused(cep.CEP_EINVAL, b, _linear(), y, x, w, BIG, dx=y)
    _refused(cep.CEP_EINVAL, b, _linear(), y, x, w, BIG, dx=x, dw=PTR + 4096)


def test_outputs_over_arrays_that_are_still_read_are_refused():
    f, b = cep.cep_linear, cep.cep_linear_backward
    x, w, y, v = (PTR + 4096 * i for i in range(4))
    for over in (dict(y=w), dict(y=x), dict(bias=y)):
        _refused(cep.CEP_EINVAL, f, _linear(), x, w, over.get("y", y), BIG, bias=over.get("bias"))
    for name in ("bias", "mul", "residual"):
        _refused(cep.CEP_EINVAL, f, _linear(), x, w, y, BIG, preact=v, **{name: v})
    _refused(cep.CEP_EINVAL, f, _linear(), x, w, y, BIG, preact=w)
    for out in ("dx", "dw", "dbias"):
        for p in (y, x, w):
            _refused(cep.CEP_EINVAL, b, _linear(), y, x, w, BIG, **{out: p})
    for name in ("mul", "preact"):
        _refused(cep.CEP_EINVAL, b, _linear(act=cep.CEP_SILU), y, x, w, BIG, dbias=v,
                 **{"preact": PTR + 5 * 4096, name: v})
    _refused(cep.CEP_EINVAL, cep.cep_expert_sort, _sort(), PTR, PTR, PTR, PTR, BIG, x=x, out_x=x)
    _refused(cep.CEP_EINVAL, cep.cep_expert_unsort, _unsort(), x, PTR, x)
    _refused(cep.CEP_EINVAL, cep.cep_expert_unsort_backward, _unsort(), x, y, PTR, None, x, None)


# --------------------------------------------------------- routed experts

def _routed(E=2, d=8, d_ff=16, top_k=2):
    from paper_2609_33252_amd import moe_block
    w = [torch.zeros(E, *n, dtype=torch.bfloat16) for n in ((d, d_ff), (d, d_ff), (d_ff, d))]
    return moe_block.RoutedExperts(top_k=top_k, w_gate=w[0], w_up=w[1], w_down=w[2])


@pytest.mark.parametrize("bad", [dict(E=0), dict(E=1025), dict(d=12), dict(d=0), dict(d=32776),
                                 dict(d_ff=4), dict(d_ff=20), dict(top_k=0), dict(top_k=17)])
def test_routed_experts_refuse_sizes_before_a_pass(bad):
    with pytest.raises(ValueError):
        _routed(**bad)


@pytest.mark.parametrize("T,k", [((1 << 17) + 1, 16), ((1 << 20) + 1, 2), ((1 << 21) + 1, 1)])
def test_routed_experts_refuse_more_rows_than_the_products_take(T, k, monkeypatch):
    r = _routed(top_k=k)
    monkeypatch.setattr(r, "_forward", lambda *a: pytest.fail("launched"))
    with pytest.raises(ValueError, match="2.21 rows"):
        r.forward(torch.zeros(T, 8, dtype=torch.bfloat16), torch.zeros(T, k, dtype=torch.int32),
                  torch.zeros(T, k))

# ------------------------------------------------------------ gate gradient

def _gate(**kw):
    return cep.make_gate(**{**dict(rows=4, n_experts=64, top_k=8, normalize=1, scale=1.0), **kw})


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=(1 << 21) + 1), dict(n_experts=0),
                                 dict(n_experts=1025), dict(top_k=0), dict(top_k=17),
                                 dict(top_k=5, n_experts=4), dict(logit_dtype=2), dict(score=2),
                                 dict(ld=63), dict(scale=float("nan")),
                                 dict(score=1, n_groups=3, topk_groups=1),
                                 dict(n_groups=8, topk_groups=4)])
def test_gate_gradient_refuses_descriptors(bad):
    _refused(cep.CEP_EINVAL, cep.cep_gate_topk_backward, _gate(**bad), PTR, PTR, PTR, 2 * PTR)


def test_gate_gradient_refuses_arguments():
    f = cep.cep_gate_topk_backward
    _refused(cep.CEP_EINVAL, f, None, PTR, PTR, PTR, 2 * PTR)
    for i in range(4):
        for wrong in (None, PTR + 2):
            _refused(cep.CEP_EINVAL, f, _gate(), *[wrong if j == i else (j + 1) * PTR
                                                   for j in range(4)])
    _refused(cep.CEP_EINVAL, f, _gate(), PTR, PTR, PTR, PTR)  # in place
    f(_gate(rows=0), None, None, None, None)


# --------------------------------------------- formulas against differences
# central differences with h = 1e-5 of functions of order 1: truncation h^2 times
# third derivatives of order 10 (1e-9), rounding 2^-53 / h of sums of order 100 (1e-9)

def _slope(f, x, v, h=1e-5):
    return float((f(x + h * v) - f(x - h * v)) / (2 * h))


@pytest.mark.parametrize("code", range(5))
@pytest.mark.parametrize("offsets", [None, [0, 2, 2, 7]])
def test_linear_gradient_formula_agrees_with_differences(code, offsets):
    g = torch.Generator().manual_seed(code)
    r = lambda *n: torch.randn(*n, generator=g, dtype=torch.float64)
    lead = () if offsets is None else (3,)
    a = dict(x=r(7, 8), w=r(*lead, 8, 16) * 0.3, bias=r(*lead, 16), mul=r(7, 16), res=r(7, 16))
    dy = r(7, 16)
    z = R.linear(**a, code=code, offsets=offsets)[0]
    grads = R.linear_grad(dy, a["x"], a["w"], z, a["mul"], code, offsets)
    grads["res"] = dy
    for name, key in (("x", "dx"), ("w", "dw"), ("bias", "db"), ("mul", "dm"), ("res", "res")):
        v = r(*a[name].shape)
        f = lambda t: (R.linear(**{**a, name: t}, code=code, offsets=offsets)[1] * dy).sum()
        assert abs(_slope(f, a[name], v) - float((grads[key] * v).sum())) < 1e-6, name


def test_unsort_gradient_formula_agrees_with_differences():
    g = torch.Generator().manual_seed(5)
    r = lambda *n: torch.randn(*n, generator=g, dtype=torch.float64)
    place = torch.tensor([[3, -1], [0, 2], [-1, -1], [1, 4]])
    ys, w, res, dy = r(5, 6), r(4, 2), r(4, 6), r(4, 6)
    dys, dw, _ = R.expert_unsort_grad(dy, ys, place, w)
    v, u = r(5, 6), r(4, 2)
    f = lambda a, b: (R.expert_unsort(a, place, b, res)[0] * dy).sum()
    assert abs(_slope(lambda z: f(z, w), ys, v) - float((dys * v).sum())) < 1e-6
    assert abs(_slope(lambda z: f(ys, z), w, u) - float((dw * u).sum())) < 1e-6
    # the sort's gradient is the way back without weights
    x, ids = r(4, 6), np.array([[1, -1], [0, 0], [-1, -1], [0, 2]])
    plan, pair, place = R.expert_sort(ids, 3)
    dxs, n = r(5, 6), int(plan[3])
    assert n == 5
    f = lambda z: (z[torch.from_numpy(pair).long() // 2] * dxs).sum()
    dx = R.expert_unsort(dxs, torch.from_numpy(place), None, None)[0]
    v = r(4, 6)
    assert abs(_slope(f, x, v) - float((dx * v).sum())) < 1e-6


@pytest.mark.parametrize("score,normalize", [("softmax", True), ("softmax", False),
                                             ("sigmoid", True), ("sigmoid", False)])
def test_gate_gradient_formula_agrees_with_differences(score, normalize):
    r = np.random.default_rng(3)
    l, v, dw = r.normal(size=(5, 9)), r.normal(size=(5, 9)), r.normal(size=(5, 3))
    l[2, 3:] = -np.inf  # as many experts as slots
    l[3, 1:] = -np.inf  # fewer
    l[4] = -np.inf      # none
    v[np.isinf(l)] = 0
    kw = dict(score=score, normalize=normalize, scale=1.7)
    ids, _ = B.gate(l, 3, **kw)
    f = lambda z: float((B.gate(z, 3, **kw)[1] * dw).sum())
    d = R.gate_grad(l, ids, dw, **kw)
    assert (d[np.isinf(l)] == 0).all()
    assert abs((f(l + 1e-5 * v) - f(l - 1e-5 * v)) / 2e-5 - (d * v).sum()) < 1e-6
