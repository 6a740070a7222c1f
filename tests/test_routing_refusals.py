"""What the choice of experts and the sorting of tokens refuse, without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2605_04478_amd import ccld, step

BAD_ARG, NULL, CAPACITY, WORKSPACE = -6, -7, -8, -12
I32, F32 = torch.int32, torch.float32


def z(*shape, dtype=F32):
    return torch.zeros(shape, dtype=dtype)


@pytest.mark.parametrize("call,word", [
    (lambda: step.route(z(4), 1), "scores has shape"), (lambda: step.route(z(4, 8, dtype=torch.float64), 1), "scores has type"),
    (lambda: step.route(z(4, 0), 1), "scores has 0 columns"), (lambda: step.route(z(4, 1025), 1), "scores has 1025 columns"),
    (lambda: step.route(z(4, 8), 0), "k is 0"), (lambda: step.route(z(4, 8), 9), "k is 9"), (lambda: step.route(z(4, 100), 65), "k is 65"),
    (lambda: step.route(z(4, 8), 2.0), "k is 2.0"), (lambda: step.route(z(4, 8), True), "k is True"), (lambda: step.route([1.0], 1), "scores is no tensor"),
    (lambda: step.route(z(4, 8), 2), "not on a GPU"),
    (lambda: step.route_grad(z(4, 2), z(4, 8), z(4, 2), z(4, 2)), "experts has type"), (lambda: step.route_grad(z(4, 3), z(4, 8), z(4, 2, dtype=I32), z(4, 2)), "dweights has shape"),
    (lambda: step.route_grad(z(4, 2), z(5, 8), z(4, 2, dtype=I32), z(4, 2)), "experts has shape"),
    (lambda: step.route_grad(z(4, 2), z(4, 8), z(4, 2, dtype=I32), z(4, 2)), "not on a GPU"),
    (lambda: step.expert_order(z(4, 2), 3), "experts has type"), (lambda: step.expert_order(z(4, dtype=I32), 3), "experts has shape"),
    (lambda: step.expert_order(z(4, 0, dtype=I32), 3), "no columns"), (lambda: step.expert_order(z(4, 2, dtype=I32), 0), "n_experts is 0"),
    (lambda: step.expert_order(z(4, 2, dtype=I32), 1025), "n_experts is 1025"), (lambda: step.expert_order(z(4, 2, dtype=I32), 3), "not on a GPU"),
    (lambda: step.dispatch(z(5, 8), z(4, 2, dtype=I32), z(3, dtype=I32)), "x has shape"), (lambda: step.dispatch(z(4, 0), z(4, 2, dtype=I32), z(3, dtype=I32)), "x has no columns"),
    (lambda: step.dispatch(z(4, 8), z(4, 2), z(3, dtype=I32)), "places has type"), (lambda: step.dispatch(z(4, 8), z(4, 65, dtype=I32), z(3, dtype=I32)), "places has 65"),
    (lambda: step.dispatch(z(4, 8), z(4, 2, dtype=I32), z(0, dtype=I32)), "offsets is empty"), (lambda: step.dispatch(z(4, 8), z(4, 2, dtype=I32), z(3)), "offsets has type"),
    (lambda: step.dispatch(z(4, 8), z(4, 2, dtype=I32), z(3, dtype=I32)), "not on a GPU"),
    (lambda: step.dispatch_grad(z(4, 8), z(4, 2, dtype=I32)), "drows has shape"), (lambda: step.dispatch_grad(z(8, 8), z(4, 2, dtype=I32)), "not on a GPU"),
    (lambda: step.combine(z(8, 8), z(4, 2, dtype=I32), z(4, 2, dtype=torch.bfloat16)), "weights has type"), (lambda: step.combine(z(7, 8), z(4, 2, dtype=I32), z(4, 2)), "y has shape"),
    (lambda: step.combine(z(8, 8), z(4, 2, dtype=I32), z(4, 3)), "weights has shape"), (lambda: step.combine(z(8, 8), z(4, 2, dtype=I32), z(4, 2)), "not on a GPU"),
    (lambda: step.combine_grad(z(4, 9), z(8, 8), z(4, 2, dtype=I32), z(4, 2), z(3, dtype=I32)), "y has shape"),
    (lambda: step.combine_grad(z(4, 8, dtype=torch.float16), z(8, 8), z(4, 2, dtype=I32), z(4, 2), z(3, dtype=I32)), "y has type"),
    (lambda: step.combine_grad(z(4, 8), z(8, 8), z(4, 2, dtype=I32), z(4, 2), z(3, dtype=I32)), "not on a GPU"),
])
def test_refuses(call, word):
    with pytest.raises(ValueError, match=word):
        call()


def _route(**change):
    at = 1 << 20
    a = dict(dtype=0, over_all=0, tokens=4, n_experts=8, k=2, scores=at, experts=at, weights=at, dweights=at, dscores=at, ldscores=8, lddscores=8)
    return step._RouteArgs(**{**a, **change})


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), BAD_ARG), (dict(tokens=-1), BAD_ARG), (dict(n_experts=0), BAD_ARG), (dict(k=0), BAD_ARG), (dict(k=9), BAD_ARG), (dict(n_experts=1025, ldscores=1025), CAPACITY),
    (dict(n_experts=100, ldscores=100, k=65), CAPACITY), (dict(tokens=1 << 31), CAPACITY), (dict(ldscores=7), BAD_ARG), (dict(scores=None), NULL), (dict(experts=None), NULL),
    (dict(weights=None), NULL), (dict(scores=1), BAD_ARG), (dict(experts=2), BAD_ARG), (dict(weights=2), BAD_ARG)])
def test_route_status(change, status):
    assert ccld.lib().ccld_route(C.addressof(_route(**change)), None) == status


@pytest.mark.parametrize("change,status", [(dict(dweights=None), NULL), (dict(dscores=None), NULL), (dict(over_all=1, scores=None), NULL), (dict(lddscores=7), BAD_ARG),
                                           (dict(dweights=2), BAD_ARG), (dict(dscores=1), BAD_ARG)])
def test_route_grad_status(change, status):
    assert ccld.lib().ccld_route_grad(C.addressof(_route(**change)), None) == status


def _order(**change):
    at = 1 << 20
    a = dict(expert_bits=32, tokens=4, k=2, n_experts=8, experts=at, places=at, offsets=at, workspace=None, workspace_bytes=0)
    return step._OrderArgs(**{**a, **change})


@pytest.mark.parametrize("change,status", [
    (dict(expert_bits=16), BAD_ARG), (dict(tokens=-1), BAD_ARG), (dict(k=0), BAD_ARG), (dict(n_experts=0), BAD_ARG), (dict(n_experts=1025), CAPACITY), (dict(tokens=1 << 31), CAPACITY),
    (dict(tokens=1 << 30, k=2), CAPACITY), (dict(experts=None), NULL), (dict(places=None), NULL), (dict(offsets=None), NULL), (dict(experts=2), BAD_ARG), (dict(places=2), BAD_ARG),
    (dict(offsets=2), BAD_ARG), (dict(tokens=1 << 20), WORKSPACE), (dict(tokens=1 << 20, workspace=(1 << 20) + 8, workspace_bytes=1 << 30), WORKSPACE)])
def test_order_status(change, status):
    assert ccld.lib().ccld_expert_order(C.addressof(_order(**change)), None) == status


@pytest.mark.parametrize("tokens", [1, 8192, 8193, 1 << 20, (1 << 30) - 1])
@pytest.mark.parametrize("n", [1, 128, 1024])
def test_order_workspace_is_small(tokens, n):
    need = C.c_uint64(0)
    assert ccld.lib().ccld_order_workspace(C.addressof(_order(tokens=tokens, n_experts=n)), C.addressof(need)) == 0
    assert need.value <= 257 * 4 * n
    assert ccld.lib().ccld_order_workspace(C.addressof(_order(tokens=tokens, n_experts=n)), None) == NULL


def _exchange(**change):
    at = 1 << 20
    a = dict(dtype=0, tokens=4, k=2, d=8, places=at, used=at, weights=at, x=at, y=at, x_out=at, y_out=at, dweights=at, ldx=8, ldy=8, ldx_out=8, ldy_out=8)
    return step._ExchangeArgs(**{**a, **change})


@pytest.mark.parametrize("call,change,status", [
    ("dispatch", dict(dtype=3), BAD_ARG), ("dispatch", dict(tokens=-1), BAD_ARG), ("dispatch", dict(k=0), BAD_ARG), ("dispatch", dict(d=0), BAD_ARG), ("dispatch", dict(k=65), CAPACITY),
    ("dispatch", dict(tokens=1 << 30), CAPACITY), ("dispatch", dict(tokens=1 << 31, k=1), CAPACITY), ("dispatch", dict(d=1 << 28, ldx=1 << 28, ldy_out=1 << 28), CAPACITY),
    ("dispatch", dict(x=None), NULL), ("dispatch", dict(y_out=None), NULL), ("dispatch", dict(used=None), NULL), ("dispatch", dict(places=None), NULL), ("dispatch", dict(ldx=7), BAD_ARG),
    ("dispatch", dict(ldy_out=7), BAD_ARG), ("dispatch", dict(x=1), BAD_ARG), ("dispatch", dict(y_out=1), BAD_ARG), ("dispatch", dict(used=2), BAD_ARG), ("dispatch", dict(places=2), BAD_ARG),
    ("dispatch_grad", dict(y=None), NULL), ("dispatch_grad", dict(x_out=None), NULL), ("dispatch_grad", dict(ldy=7), BAD_ARG), ("dispatch_grad", dict(ldx_out=7), BAD_ARG),
    ("combine", dict(weights=None), NULL), ("combine", dict(weights=2), BAD_ARG), ("combine", dict(y=1), BAD_ARG), ("combine", dict(x_out=1), BAD_ARG),
    ("combine_grad", dict(y=None), NULL), ("combine_grad", dict(x=None), NULL), ("combine_grad", dict(used=None), NULL), ("combine_grad", dict(dweights=2), BAD_ARG),
    ("combine_grad", dict(ldy=7), BAD_ARG), ("combine_grad", dict(dtype=2, y=2), BAD_ARG)])
def test_exchange_status(call, change, status):
    assert getattr(ccld.lib(), "ccld_" + call)(C.addressof(_exchange(**change)), None) == status


def test_nothing_at_all():
    L = ccld.lib()
    for name in ("route", "route_grad", "expert_order", "dispatch", "dispatch_grad", "combine", "combine_grad"):
        assert getattr(L, "ccld_" + name)(None, None) == NULL
        native = getattr(step._native(), name)
        assert native() is None and native(None, 1, 2.0) is None
    need = C.c_uint64(0)
    assert L.ccld_order_workspace(None, C.addressof(need)) == NULL
