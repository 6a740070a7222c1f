"""What the operators of a training step refuse, without a GPU: shapes and types in Python, sizes and pointers at the C ABI."""
import ctypes as C

import pytest
import torch

from paper_2605_04478_amd import ccld, step

BF = torch.bfloat16
BAD_ARG, NULL, CAPACITY, WORKSPACE = -6, -7, -8, -12


def _experts(**change):
    t = dict(x=torch.zeros(4, 8, dtype=BF), w=torch.zeros(2, 16, 8, dtype=BF), offsets=torch.zeros(3, dtype=torch.int32))
    t.update(change)
    return t


@pytest.mark.parametrize("change,word", [
    (dict(x=torch.zeros(4, 9, dtype=BF)), "x has shape"),
    (dict(x=torch.zeros(4, 2, 8, dtype=BF)), "x has shape"),
    (dict(x=torch.zeros(4, 8, dtype=torch.float16)), "x has type"),
    (dict(w=torch.zeros(2, 16, 8)), "w has type"),
    (dict(w=torch.zeros(16, 8, dtype=BF)), "w has shape"),
    (dict(offsets=torch.zeros(2, dtype=torch.int32)), "offsets has shape"),
    (dict(offsets=torch.zeros(3)), "offsets has type"),
    (dict(x=[1.0]), "x is no tensor"),
    (dict(), "not on a GPU"),
])
def test_expert_product_refuses(change, word):
    with pytest.raises(ValueError, match=word):
        step.expert_product(**_experts(**change))
    with pytest.raises(ValueError, match=word):
        step.expert_product_grad(torch.zeros(4, 16, dtype=BF), **_experts(**change))


def _expert_args(**change):
    """Arguments that are right but for the changes; the pointers are never followed."""
    at = 1 << 20
    a = dict(dtype=0, offsets_bits=32, rows=4, k=8, n=16, n_experts=2, x=at, w=at, offsets=at, dy=at, y=at, dx=at, dw=at,
             ldx=8, ldw=8, expert_stride=128, lddy=16, ldy=16, lddx=8)
    a.update(change)
    return step._ExpertArgs(**a)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), BAD_ARG), (dict(dtype=-1), BAD_ARG), (dict(offsets_bits=16), BAD_ARG), (dict(rows=-1), BAD_ARG),
    (dict(k=0), BAD_ARG), (dict(n=0), BAD_ARG), (dict(n_experts=0), BAD_ARG), (dict(ldx=7), BAD_ARG), (dict(ldw=7), BAD_ARG),
    (dict(ldy=15), BAD_ARG), (dict(expert_stride=-1), BAD_ARG), (dict(rows=1 << 31), CAPACITY), (dict(ldx=1 << 40), CAPACITY),
    (dict(ldw=1 << 40), CAPACITY), (dict(k=1 << 23, ldx=1 << 23, ldw=1 << 23), CAPACITY), (dict(n_experts=1 << 30), CAPACITY),
    (dict(x=None), NULL), (dict(w=None), NULL), (dict(offsets=None), NULL), (dict(y=None), NULL), (dict(offsets=2), BAD_ARG),
    (dict(x=1), BAD_ARG), (dict(k=8192, ldx=8192, ldw=8192), WORKSPACE),
])
def test_expert_product_status(change, status):
    assert ccld.lib().ccld_expert_product(C.addressof(_expert_args(**change)), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(dy=None), NULL), (dict(x=None), NULL), (dict(lddy=15), BAD_ARG), (dict(lddx=7), BAD_ARG), (dict(dw=3), BAD_ARG),
    (dict(lddy=1 << 40), CAPACITY), (dict(rows=1 << 20), WORKSPACE),
])
def test_expert_gradient_status(change, status):
    assert ccld.lib().ccld_expert_product_grad(C.addressof(_expert_args(**change)), None) == status


def test_null_arguments():
    L = ccld.lib()
    need = C.c_uint64(0)
    assert L.ccld_vocab_loss(None, None) == L.ccld_vocab_loss_grad(None, None) == L.ccld_vocab_workspace(None, 0, C.addressof(need)) == NULL
    assert L.ccld_norm_residual(None, None) == L.ccld_norm_residual_grad(None, None) == L.ccld_norm_workspace(None, C.addressof(need)) == NULL
    assert L.ccld_expert_product(None, None) == NULL and L.ccld_expert_product_grad(None, None) == NULL
    assert L.ccld_expert_workspace(None, 0, C.addressof(need)) == NULL
    assert L.ccld_expert_workspace(C.addressof(_expert_args()), 0, None) == NULL
    assert L.ccld_expert_workspace(C.addressof(_expert_args()), 0, C.addressof(need)) == 0 and need.value == 0
    a = _expert_args(rows=64, k=8192, ldx=8192, ldw=8192)
    assert L.ccld_expert_workspace(C.addressof(a), 0, C.addressof(need)) == 0 and need.value >= 2 * 4 * 64 * 16
    a.workspace, a.workspace_bytes = (1 << 20) + 8, need.value           # misaligned
    assert L.ccld_expert_product(C.addressof(a), None) == WORKSPACE


# ---- the vocabulary's loss ----------------------------------------------------------------------------------------------
def _vocab(**change):
    t = dict(h=torch.zeros(4, 8, dtype=BF), w=torch.zeros(10, 8, dtype=BF), labels=torch.zeros(4, dtype=torch.int64))
    t.update(change)
    return t


@pytest.mark.parametrize("change,word", [
    (dict(h=torch.zeros(4, 9, dtype=BF)), "h has shape"),
    (dict(h=torch.zeros(2, 2, 8, dtype=BF)), "h has shape"),
    (dict(h=torch.zeros(4, 8)), "h has type"),
    (dict(w=torch.zeros(10, 8, dtype=torch.float64)), "w has type"),
    (dict(w=torch.zeros(0, 8, dtype=BF)), "no size may be zero"),
    (dict(labels=torch.zeros(5, dtype=torch.int64)), "labels has shape"),
    (dict(labels=torch.zeros(4)), "labels has type"),
    (dict(), "not on a GPU"),
])
def test_vocab_loss_refuses(change, word):
    with pytest.raises(ValueError, match=word):
        step.vocab_loss(**_vocab(**change))
    with pytest.raises(ValueError, match=word):
        step.vocab_loss_grad(torch.zeros(4), lse=torch.zeros(4), **_vocab(**change))


def _vocab_args(**change):
    at = 1 << 20
    a = dict(dtype=0, label_bits=64, rows=4, d=8, vocab=10, h=at, w=at, labels=at, dloss=at, loss=at, lse=at, dh=at, dw=at, ldh=8,
             ldw=8, dloss_stride=1, lddh=8, lddw=8, workspace=at, workspace_bytes=1 << 30)
    a.update(change)
    return step._VocabArgs(**a)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), BAD_ARG), (dict(label_bits=8), BAD_ARG), (dict(rows=-1), BAD_ARG), (dict(d=0), BAD_ARG), (dict(vocab=0), BAD_ARG),
    (dict(ldh=7), BAD_ARG), (dict(ldw=7), BAD_ARG), (dict(rows=1 << 31), CAPACITY), (dict(vocab=1 << 31), CAPACITY),
    (dict(ldw=1 << 40), CAPACITY), (dict(rows=1 << 30, vocab=1 << 30), CAPACITY), (dict(h=None), NULL), (dict(w=None), NULL),
    (dict(labels=None), NULL), (dict(loss=None), NULL), (dict(lse=None), NULL), (dict(labels=4), BAD_ARG), (dict(loss=2), BAD_ARG),
    (dict(workspace=None), WORKSPACE), (dict(workspace=(1 << 20) + 16), WORKSPACE), (dict(workspace_bytes=100), WORKSPACE),
])
def test_vocab_loss_status(change, status):
    assert ccld.lib().ccld_vocab_loss(C.addressof(_vocab_args(**change)), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(dloss=None), NULL), (dict(lse=None), NULL), (dict(dloss_stride=-1), BAD_ARG), (dict(lddh=7), BAD_ARG), (dict(lddw=7), BAD_ARG),
    (dict(dw=1), BAD_ARG), (dict(dloss=6), BAD_ARG), (dict(workspace_bytes=1000), WORKSPACE),
])
def test_vocab_gradient_status(change, status):
    assert ccld.lib().ccld_vocab_loss_grad(C.addressof(_vocab_args(**change)), None) == status


# ---- the norms ------------------------------------------------------------------------------------------------------------
def _norm(**change):
    t = dict(h=torch.zeros(6, 8), b=torch.zeros(6, 8), gate=torch.zeros(3, 8), w_post=torch.zeros(8), w_pre=torch.zeros(8))
    t.update(change)
    return t


@pytest.mark.parametrize("change,word", [
    (dict(b=torch.zeros(6, 9)), "b has shape"),
    (dict(b=torch.zeros(6, 8, dtype=BF)), "b has type"),
    (dict(h=torch.zeros(6, 8, dtype=torch.float64)), "h has type"),
    (dict(h=torch.zeros(6, 20000), b=torch.zeros(6, 20000), gate=None, w_post=torch.zeros(20000), w_pre=torch.zeros(20000)), "columns"),
    (dict(h=torch.zeros(6, 0), b=torch.zeros(6, 0), gate=None, w_post=torch.zeros(0), w_pre=torch.zeros(0)), "columns"),
    (dict(gate=torch.zeros(4, 8)), "share 4 rows of gate"),
    (dict(gate=torch.zeros(0, 8)), "share 0 rows of gate"),
    (dict(gate=torch.zeros(8)), "gate has shape"),
    (dict(w_post=torch.zeros(1, 8)), "w_post has shape"),
    (dict(w_pre=torch.zeros(8, dtype=BF)), "w_pre has type"),
    (dict(), "not on a GPU"),
])
def test_norm_residual_refuses(change, word):
    t = _norm(**change)
    with pytest.raises(ValueError, match=word):
        step.norm_residual(**t)
    with pytest.raises(ValueError, match=word):
        step.norm_residual_grad(t["h"], t["h"], *t.values(), torch.zeros(6), torch.zeros(6))


def test_norm_residual_refuses_a_negative_eps():
    with pytest.raises(ValueError, match="eps"):
        step.norm_residual(**_norm(), eps=-1.0)


def _norm_args(**change):
    at = 1 << 20
    a = dict(dtype=2, scale=1.0, eps=1e-6, rows=6, d=8, groups=3, workspace=at, workspace_bytes=1 << 30)
    a.update({n: at for n in ("h", "b", "gate", "w_post", "w_pre", "h_out", "u", "rstd_post", "rstd_pre", "dh_out", "du", "dh", "db",
                              "dgate", "dw_post", "dw_pre")})
    a.update({n: 8 for n in ("ldh", "ldb", "ldgate", "ldh_out", "ldu", "lddh_out", "lddu", "lddh", "lddb")})
    a.update(change)
    return step._NormArgs(**a)


SHARED = [
    (dict(dtype=3), BAD_ARG), (dict(rows=-6), BAD_ARG), (dict(d=0), BAD_ARG), (dict(groups=0), BAD_ARG), (dict(groups=4), BAD_ARG),
    (dict(d=20000), CAPACITY), (dict(rows=3 << 31), CAPACITY), (dict(eps=-1.0), BAD_ARG), (dict(eps=float("nan")), BAD_ARG),
    (dict(h=None), NULL), (dict(b=None), NULL), (dict(w_post=None), NULL), (dict(w_pre=None), NULL), (dict(rstd_pre=None), NULL),
    (dict(ldh=7), BAD_ARG), (dict(ldb=7), BAD_ARG), (dict(ldgate=7), BAD_ARG), (dict(h=2), BAD_ARG), (dict(rstd_post=2), BAD_ARG),
]


@pytest.mark.parametrize("change,status", SHARED + [(dict(h_out=None), NULL), (dict(u=None), NULL), (dict(ldu=7), BAD_ARG), (dict(u=2), BAD_ARG)])
def test_norm_residual_status(change, status):
    assert ccld.lib().ccld_norm_residual(C.addressof(_norm_args(**change)), None) == status


@pytest.mark.parametrize("change,status", SHARED + [
    (dict(dh=None), NULL), (dict(dw_pre=None), NULL), (dict(lddh=7), BAD_ARG), (dict(lddu=7), BAD_ARG), (dict(du=2), BAD_ARG),
    (dict(workspace=None), WORKSPACE), (dict(workspace_bytes=8), WORKSPACE), (dict(workspace=(1 << 20) + 4), WORKSPACE)])
def test_norm_gradient_status(change, status):
    assert ccld.lib().ccld_norm_residual_grad(C.addressof(_norm_args(**change)), None) == status
