"""What the log probabilities of tokens refuse, without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2605_04478_amd import ccld, step

BAD_ARG, NULL, CAPACITY, WORKSPACE = -6, -7, -8, -12
NAN, INF = float("nan"), float("inf")


def z(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


T = z(4, dtype=torch.int64)


@pytest.mark.parametrize("args,word", [
    ((z(4), T), "logits has shape"), ((z(4, 8, dtype=torch.float64), T), "logits has type"), ((z(4, 0), T), "logits has no columns"), ((z(4, 8), z(4)), "tokens has type"),
    ((z(4, 8), z(5, dtype=torch.int64)), "tokens has shape"), ((z(4, 8), T, 0.0), "temperature is 0.0"), ((z(4, 8), T, -1), "temperature is -1"), ((z(4, 8), T, NAN), "temperature is nan"),
    ((z(4, 8), T, INF), "temperature is inf"), ((z(4, 8), T, "x"), "temperature is 'x'"), (([1.0], T), "logits is no tensor"), ((z(4, 8), T), "not on a GPU")])
def test_token_logprobs_refuses(args, word):
    with pytest.raises(ValueError, match=word):
        step.token_logprobs(*args)
    if len(args) < 4:
        f = z(4)
        with pytest.raises(ValueError, match=word):
            step.token_logprobs_grad(f, f, args[0], args[1], f, f, *args[2:])


@pytest.mark.parametrize("change,word", [(dict(dlogp=z(5)), "dlogp has shape"), (dict(dentropy=z(4).half()), "dentropy has type"), (dict(lse=None), "lse is no tensor"),
                                         (dict(entropy=z(3)), "entropy has shape"), (dict(dlogp=None, dentropy=None), "not on a GPU")])
def test_gradient_refuses(change, word):
    f = z(4)
    with pytest.raises(ValueError, match=word):
        step.token_logprobs_grad(**{**dict(dlogp=f, dentropy=f, logits=z(4, 8), tokens=T, lse=f, entropy=f), **change})


def _args(**change):
    at = 1 << 20
    a = dict(dtype=0, token_bits=64, temperature=1.0, top=2, rows=4, vocab=8, logits=at, tokens=at, logp=at, entropy=at, lse=at, top_ids=at, top_logp=at, dlogp=at, dentropy=at, dlogits=at,
             ldlogits=8, lddlogits=8, dlogp_stride=1, dentropy_stride=1, workspace=None, workspace_bytes=0)
    return step._LogprobArgs(**{**a, **change})


BOTH = [(dict(dtype=3), BAD_ARG), (dict(token_bits=16), BAD_ARG), (dict(rows=-1), BAD_ARG), (dict(vocab=0), BAD_ARG), (dict(temperature=0.0), BAD_ARG), (dict(temperature=NAN), BAD_ARG),
        (dict(temperature=INF), BAD_ARG), (dict(temperature=1e-20), BAD_ARG), (dict(rows=1 << 31), CAPACITY), (dict(vocab=1 << 31, ldlogits=1 << 31, lddlogits=1 << 31), CAPACITY), (dict(logits=None), NULL),
        (dict(tokens=None), NULL), (dict(entropy=None), NULL), (dict(lse=None), NULL), (dict(ldlogits=7), BAD_ARG), (dict(logits=1), BAD_ARG), (dict(tokens=4), BAD_ARG), (dict(lse=2), BAD_ARG)]


@pytest.mark.parametrize("change,status", BOTH + [(dict(top=-1), BAD_ARG), (dict(top=65), BAD_ARG), (dict(logp=None), NULL), (dict(top_ids=None), NULL), (dict(top_logp=None), NULL), (dict(top_ids=2), BAD_ARG)])
def test_token_logprobs_status(change, status):
    assert ccld.lib().ccld_token_logprobs(C.addressof(_args(**change)), None) == status


@pytest.mark.parametrize("change,status", BOTH + [(dict(dlogits=None), NULL), (dict(lddlogits=7), BAD_ARG), (dict(dlogits=1), BAD_ARG), (dict(dlogp=2), BAD_ARG)])
def test_gradient_status(change, status):
    assert ccld.lib().ccld_token_logprobs_grad(C.addressof(_args(**change)), None) == status


@pytest.mark.parametrize("rows", [0, 1, 3, 100, 513, 5000, (1 << 31) - 1])
@pytest.mark.parametrize("vocab", [1, 1000, 50021, 128000, 1 << 20, (1 << 31) - 1])
@pytest.mark.parametrize("dtype", [0, 2])
def test_workspace_is_small(rows, vocab, dtype):
    """64 parts of a row at most, each with three sums and `top` numbers and words, in as many as 4,096 workgroups."""
    need = C.c_uint64(9)
    assert ccld.lib().ccld_logprob_workspace(C.addressof(_args(rows=rows, vocab=vocab, ldlogits=vocab, dtype=dtype, top=64)), C.addressof(need)) == 0
    assert need.value <= min(64 * rows, 4096) * (12 + 8 * 64) + 3 * 256
    if need.value:
        a = _args(rows=rows, vocab=vocab, ldlogits=vocab, dtype=dtype, top=64, workspace=1 << 20, workspace_bytes=need.value - 1)
        assert ccld.lib().ccld_token_logprobs(C.addressof(a), None) == WORKSPACE


def test_top_is_checked():
    for top in (-1, 65, 1.0, True):
        with pytest.raises(ValueError, match="top is|not on a GPU"):
            step.token_logprobs(z(4, 100), T, 1.0, top)
    assert ccld.lib().ccld_token_logprobs(None, None) == ccld.lib().ccld_token_logprobs_grad(None, None) == NULL
    need = C.c_uint64(9)
    assert ccld.lib().ccld_logprob_workspace(C.addressof(_args()), C.addressof(need)) == 0 and ccld.lib().ccld_logprob_workspace(None, C.addressof(need)) == NULL
