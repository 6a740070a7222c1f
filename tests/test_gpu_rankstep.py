"""A rank's step on the GPU: its gradients against a step in 64 bits, and the whole way to the rank that the analyzer names."""
import numpy as np
import pytest
import torch

from paper_2605_04478_amd import rankstep

pytestmark = pytest.mark.gpu
SPEC = rankstep.StepSpec(d=96, hidden=128, experts=4, layers=2, vocab=300)


def _in_64_bits(work, h, offsets, labels):
    s, ends = work.spec, offsets.tolist()
    leaves = [w.detach().double().cpu().requires_grad_() for w in work.weights()]
    h, labels = h.double().cpu(), labels.cpu()
    u = h
    for k in range(s.layers):
        up, down, gate, post, pre = leaves[5 * k:5 * k + 5]
        block = torch.cat([torch.nn.functional.silu(u[a:b] @ up[e].t()) @ down[e].t() for e, (a, b) in enumerate(zip(ends, ends[1:]))])
        h = s.scale * h + gate * (block / torch.sqrt((block ** 2).mean(1, keepdim=True) + s.eps) * post)
        u = h / torch.sqrt((h ** 2).mean(1, keepdim=True) + s.eps) * pre
    used = labels >= 0
    z = u[used] @ leaves[-1].t()
    loss = (torch.logsumexp(z, 1) - z.gather(1, labels[used][:, None])[:, 0]).sum() / used.sum().clamp(min=1)
    return loss.detach(), torch.autograd.grad(loss, leaves)


@pytest.mark.parametrize("load,masked", [((30, 0, 50, 17), 0.3), ((1, 1, 1, 1), 0.0), ((200, 300, 0, 0), 0.9)], ids=str)
def test_step_against_64_bits(load, masked):
    work = rankstep.RankStep(SPEC)
    batch = work.batch(load, seed=3, masked=masked)
    loss, grads = work.gradients(*batch)
    want_loss, want = _in_64_bits(work, *batch)
    # a value passes 5 roundings to 8 bits in a layer's forward pass, 6 in its backward pass and 3 in the loss: at most 25 halves of a step
    # of 2^-7, each of the size of what it is a part of
    bound = 25 * 2.0 ** -8
    assert abs(float(loss) - float(want_loss)) <= bound * max(1.0, abs(float(want_loss)))
    for w, g, x in zip(work.weights(), grads, want):
        assert g.shape == w.shape and g.dtype == w.dtype
        assert float((g.double().cpu() - x).norm()) <= bound * float(x.norm()) + 1e-12, tuple(w.shape)


def test_more_rows_take_longer():
    work = rankstep.RankStep(rankstep.StepSpec(d=512, hidden=1024, experts=4, layers=1, vocab=8000))
    few, many = work.measure([rankstep.even_load(256, 4), rankstep.even_load(16384, 4)], repeats=3)
    assert 0 < few < many
    with pytest.raises(ValueError, match="load"):
        work.batch([1, 2, 3])


def test_command_names_the_busy_rank(capsys):
    assert rankstep.main(["--ranks", "6", "--busy-rank", "4", "--rows", "2048", "--times", "4", "--slots", "30"]) == 0
    assert "rank 4" in capsys.readouterr().out
