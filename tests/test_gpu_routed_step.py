"""A whole step of a rank: its gradients against a step in 64 bits, the optimizer, the evaluation and the command."""
import pytest
import torch

from paper_2605_04478_amd import rankstep, step

pytestmark = pytest.mark.gpu
SPEC = rankstep.StepSpec(d=96, hidden=128, experts=5, layers=2, vocab=300)


def _in_64_bits(work, chosen, h, labels):
    """The same step with the experts that were chosen: (loss, gradients)."""
    leaves = [w.detach().double().cpu().requires_grad_() for w in work.weights()]
    h, labels = h.double().cpu(), labels.cpu()
    u = h
    for k in range(work.spec.layers):
        up, down, gate, post, pre, router = leaves[6 * k:6 * k + 6]
        at = chosen[k].long().cpu()
        p = torch.softmax((u @ router.t()).gather(1, at), 1)
        each = torch.stack([torch.stack([torch.nn.functional.silu(u[t] @ up[e].t()) @ down[e].t() for e in at[t]]) for t in range(len(u))])
        block = (p[..., None] * each).sum(1)
        h = work.spec.scale * h + gate * (block / torch.sqrt((block ** 2).mean(1, keepdim=True) + work.spec.eps) * post)
        u = h / torch.sqrt((h ** 2).mean(1, keepdim=True) + work.spec.eps) * pre
    used = labels >= 0
    z = u[used] @ leaves[-1].t()
    loss = (torch.logsumexp(z, 1) - z.gather(1, labels[used][:, None])[:, 0]).sum() / used.sum().clamp(min=1)
    return loss.detach(), torch.autograd.grad(loss, leaves)


@pytest.mark.parametrize("choices", [1, 2, 5])
@pytest.mark.parametrize("dtype,half", [(torch.bfloat16, 2.0 ** -8), (torch.float16, 2.0 ** -11)], ids=str)
def test_gradients_against_64_bits(choices, dtype, half, monkeypatch):
    work = rankstep.RoutedStep(SPEC, choices, dtype)
    h, labels = work.batch([20, 0, 40, 13, 7], seed=3, masked=0.3)
    chosen, route = [], step.route
    monkeypatch.setattr(step, "route", lambda *a: chosen.append(route(*a)) or chosen[-1])
    loss, grads = work.gradients(h, labels)
    want_loss, want = _in_64_bits(work, [e for e, _ in chosen], h, labels)
    # a value passes 7 roundings in a layer's forward pass, 9 in its backward pass and 3 in the loss: at most 35, each of half a step of what it is a part of (and of
    # subnormal numbers' in half precision); a router's gradient is a difference of what its experts' rows say, each of which is up to twice as large
    bound = 35 * half
    assert abs(float(loss) - float(want_loss)) <= bound * max(1.0, abs(float(want_loss)))
    for i, (w, g, x) in enumerate(zip(work.weights(), grads, want)):
        assert g.shape == w.shape and g.dtype == w.dtype
        times = 2 if i % 6 == 5 and i < 6 * SPEC.layers else 1
        assert float((g.double().cpu() - x).norm()) <= times * bound * float(x.norm()) + 35 * 2.0 ** -25 * x.numel() ** 0.5, i


@pytest.mark.parametrize("bits", [32, 8])
def test_a_whole_step_updates_the_weights(bits):
    work = rankstep.RoutedStep(SPEC, 2, bits=bits)
    batch = work.batch([50, 0, 10, 3, 1], masked=0.2)
    before = [w.detach().clone() for w in work.weights()]
    _, grads = work.gradients(*batch)
    loss = work.take(*batch)
    assert torch.isfinite(loss) and int(work.optimizer.state["count"]) == 1
    at = 0
    for w, old, g in zip(work.weights(), before, grads):
        # the first step: lr against the gradient's sign where it is not next to eps, and the decay
        master = work.optimizer.state["master"][at:at + w.numel()].view_as(w)
        at += -(-w.numel() // step.ADAMW_BLOCK) * step.ADAMW_BLOCK
        want = old.double() * (1 - 1e-3 * 0.1) - 1e-3 * g.double() / (g.double().abs() + 1e-8)
        assert float((master.double() - want).abs().max()) <= 2.0 ** -22 * float(old.abs().max()) + 1e-3 * 2.0 ** -18
        assert torch.equal(w.detach(), master.to(w.dtype))
    for _ in range(3):
        loss = work.take(*batch)
    assert torch.isfinite(loss) and all(torch.isfinite(w).all() for w in work.weights())


def test_evaluation_says_what_the_loss_says():
    work = rankstep.RoutedStep(SPEC, 2, torch.float16)
    h, labels = work.batch([30, 1, 0, 9, 20], masked=0.25)
    logp, entropy, lse, ids, best = work.evaluate(h, labels, top=3)
    used = labels >= 0
    mean = -logp[used].double().mean()
    z = lse.abs().max() + 10
    # logits are rounded to half precision for one of them
    assert abs(float(mean) - float(work.loss(h, labels).detach())) <= 2 * 2.0 ** -11 * float(z)
    assert not logp[~used].any() and (entropy > 0).all() and ids.shape == (60, 3) and (best[:, 0] >= best[:, 2]).all()


def test_command_with_choices(capsys):
    assert rankstep.main(["--ranks", "6", "--busy-rank", "4", "--rows", "1024", "--times", "4", "--slots", "30", "--choices", "2"]) == 0
    assert "rank 4" in capsys.readouterr().out
    with pytest.raises(SystemExit):
        rankstep.main(["--choices", "9"])
