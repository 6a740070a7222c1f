"""The optimizer's call holds the memory that it was given until its work has been enqueued, whatever other threads do to the lists and the dict meanwhile."""
import contextlib
import gc
import threading
import weakref

import pytest
import torch

from paper_2605_04478_amd import step


class Declines:
    def __getattr__(self, _):
        return lambda *a: None


@pytest.mark.parametrize("bits", [32, 8])
def test_python_holds_what_it_took(bits, monkeypatch):
    """Without a GPU: the lists and the dict are emptied where the library would be called with their tensors' addresses."""
    monkeypatch.setattr(step, "_calls", Declines())
    monkeypatch.setattr(step, "_on_gpu", lambda first, *others: first.device)
    monkeypatch.setattr(step, "_current", lambda device: contextlib.nullcontext())
    params, grads = [torch.zeros(300, dtype=torch.bfloat16), torch.zeros(7, dtype=torch.bfloat16)], [torch.zeros(300), torch.zeros(7)]
    state = step.adamw_state(params, bits, True)
    kept = {name: (weakref.ref(t), t.data_ptr()) for name, t in state.items()}
    others = [weakref.ref(t) for t in params + grads]
    called = []

    def call(fn, args, device):
        state.clear()
        params.clear()
        grads.clear()
        gc.collect()
        assert all(ref() is not None for ref, _ in kept.values()) and all(ref() is not None for ref in others)
        assert all(getattr(args, name) == at for name, (_, at) in kept.items())
        called.append(fn.__name__)
    monkeypatch.setattr(step, "_call", call)
    step.adamw(params, grads, state, 1e-3)
    assert called == ["ccld_adamw"]


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
def test_entries_replaced_by_another_thread(native, monkeypatch):
    """One thread takes steps, another replaces the state's entries and takes their memory for tensors of its own, which stay as they are."""
    dev = "cuda:0"
    if not native:
        step._native()
        monkeypatch.setattr(step, "_calls", Declines())
    n = 1 << 16
    params, grads = [torch.zeros(n, device=dev)], [torch.ones(n, device=dev)]
    state = step.adamw_state(params)
    own, done = [], threading.Event()

    def replace():
        k = 0
        while not done.is_set() and k < 2000:
            name = ("m", "v")[k % 2]
            state[name] = state[name].clone()
            own.append(torch.full((n,), 7.0, device=dev))
            k += 1
    other = threading.Thread(target=replace)
    other.start()
    try:
        for _ in range(500):
            step.adamw(params, grads, state, 1e-3)
    finally:
        done.set()
        other.join()
    assert int(state["count"]) == 500 and own
    assert all(bool((t == 7.0).all()) for t in own)
