"""What the optimizer refuses, without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2605_04478_amd import ccld, step

BAD_ARG, NULL, CAPACITY, WORKSPACE = -6, -7, -8, -12
F32 = torch.float32


def _state(total=512, **change):
    return {"count": torch.zeros(1, dtype=torch.int64), "m": torch.zeros(total), "v": torch.zeros(total), **change}


def _step(params=None, grads=None, state=None, lr=1e-3, **more):
    params = [torch.zeros(300)] if params is None else params
    grads = [torch.zeros(300)] if grads is None else grads
    step.adamw(params, grads, _state() if state is None else state, lr, **more)


base = torch.zeros(600)


@pytest.mark.parametrize("args,word", [
    (dict(params=torch.zeros(3)), "params is no list"), (dict(params=[1.0]), r"params\[0\] is no tensor"), (dict(params=[torch.zeros(300, dtype=torch.float64)]), r"params\[0\] has type"),
    (dict(params=[torch.zeros(10), torch.zeros(10).half()], grads=[None, None]), "one call takes one type"), (dict(params=[base[::2]]), "not contiguous"),
    (dict(params=[base[:300], base[299:]], grads=[None, None]), r"params\[0\] and params\[1\] share memory"), (dict(params=[base, base], grads=[None, None]), "share memory"),
    (dict(grads=[]), "grads is no list of 1"), (dict(grads=None, state=[]), "state is no dict"), (dict(grads=[torch.zeros(299)]), r"grads\[0\] has shape"),
    (dict(grads=[torch.zeros(300).half()]), r"grads\[0\] has type"), (dict(grads=[1.0]), r"grads\[0\] is no tensor"),
    (dict(params=[torch.zeros(200).half(), torch.zeros(200).half()], grads=[torch.zeros(200).half(), torch.zeros(200)]), "others"),
    (dict(state={}), "count is no tensor"), (dict(state=_state(256)), "m has shape"), (dict(state=_state(v=torch.zeros(512).half())), "v has type"),
    (dict(state=_state(m=torch.zeros(512).to(torch.float8_e4m3fn), v=torch.zeros(512).to(torch.float8_e5m2))), "m_scale is no tensor"),
    (dict(state=_state(master=torch.zeros(512))), "masters are for 16-bit"), (dict(state=_state(m=torch.zeros(1024)[::2])), "m is not contiguous"),
    (dict(lr=float("nan")), "lr is nan"), (dict(lr="x"), "lr is 'x'"), (dict(betas=0.9), "betas is 0.9"), (dict(betas=(0.9, 1.0)), "betas is"), (dict(betas=(-0.1, 0.9)), "betas is"), (dict(eps=-1.0), "eps is -1"),
    (dict(weight_decay=float("inf")), "weight_decay is inf"), (dict(scale=torch.zeros(2)), "scale has shape"), (dict(scale=torch.zeros(1).half()), "scale has type"), (dict(scale="a"), "scale is 'a'"),
    (dict(seed=0.5), "seed is 0.5"), (dict(), "not on a GPU"),
])
def test_adamw_refuses(args, word):
    with pytest.raises(ValueError, match=word):
        _step(**args)


@pytest.mark.parametrize("args,word", [
    (dict(params=[]), "params is empty"), (dict(params=[torch.zeros(3)], bits=16), "bits is 16"), (dict(params=[torch.zeros(3)], masters=True), "masters are for 16-bit"),
    (dict(params=[base, base[5:]]), "share memory"), (dict(params=[torch.zeros(3)]), "not on a GPU")])
def test_state_refuses(args, word):
    with pytest.raises(ValueError, match=word):
        step.adamw_state(**args)


def _args(tensor=(1 << 20, 1 << 20, 300, 0), n_tensors=1, **change):
    at = 1 << 20
    table = (step._AdamwTensor * 1)(step._AdamwTensor(*tensor))
    a = dict(dtype=0, grad_dtype=0, bits=32, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, scale=1.0, scale_by=None, seed=0, tensors=C.addressof(table), n_tensors=n_tensors,
             total=512, count=at, m=at, v=at, m_scale=at, v_scale=at, master=None, workspace=at, workspace_bytes=256)
    args = step._AdamwArgs(**{**a, **change})
    args.keep = table
    return args


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), BAD_ARG), (dict(grad_dtype=1), BAD_ARG), (dict(bits=16), BAD_ARG), (dict(lr=NAN), BAD_ARG), (dict(weight_decay=INF), BAD_ARG), (dict(scale=NAN), BAD_ARG), (dict(eps=-1.0), BAD_ARG),
    (dict(eps=NAN), BAD_ARG), (dict(beta1=1.0), BAD_ARG), (dict(beta2=-0.5), BAD_ARG), (dict(beta2=NAN), BAD_ARG), (dict(n_tensors=-1), BAD_ARG), (dict(total=500), BAD_ARG), (dict(total=-256), BAD_ARG),
    (dict(dtype=2, grad_dtype=2, master=1 << 20), BAD_ARG), (dict(total=1 << 41), CAPACITY), (dict(count=None), NULL), (dict(tensors=None), NULL), (dict(m=None), NULL), (dict(v=None), NULL),
    (dict(bits=8, m_scale=None), NULL), (dict(bits=8, v_scale=None), NULL), (dict(count=4), BAD_ARG), (dict(m=2), BAD_ARG), (dict(scale_by=2), BAD_ARG), (dict(workspace=None), WORKSPACE),
    (dict(workspace_bytes=128), WORKSPACE), (dict(workspace=(1 << 20) + 8), WORKSPACE), (dict(tensor=(None, 1 << 20, 300, 0)), NULL), (dict(tensor=(1 << 20, None, 300, 0)), NULL),
    (dict(tensor=(1, 1 << 20, 300, 0)), BAD_ARG), (dict(tensor=(1 << 20, 1, 300, 0)), BAD_ARG), (dict(tensor=(1 << 20, 1 << 20, -1, 0)), BAD_ARG), (dict(tensor=(1 << 20, 1 << 20, 300, 100)), BAD_ARG),
    (dict(tensor=(1 << 20, 1 << 20, 300, 256)), BAD_ARG), (dict(tensor=(1 << 20, 1 << 20, 300, -256)), BAD_ARG), (dict(tensor=(1 << 20, 1 << 20, 1 << 62, 256)), BAD_ARG)])
def test_adamw_status(change, status):
    assert ccld.lib().ccld_adamw(C.addressof(_args(**change)), None) == status
    assert ccld.lib().ccld_adamw(None, None) == NULL
