"""A rank's training step, computed on this card, and the trace of a job whose ranks take it.

The analysis names a rank whose computation is slow (Section 2.2, S1).  Its card may be slow, or it was given more work: what its work takes on a
card that is known to be sound tells, beside what it took in the job.  `RankStep` is a step's computation (experts, norms with gate and
residual scale, the vocabulary's loss; forward and backward) with the operators of `step`, `measure` times it on this card for given loads, and
`trace` lets the ranks of a job compute for so long between their collectives, so that the analyzer sees what these times would do to a job.

    python -m paper_2605_04478_amd.rankstep --ranks 16 --busy-rank 5 --took-us 9000
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass, replace
from typing import List, Sequence

import numpy as np
import torch

from . import step, tracegen as tg


@dataclass(frozen=True)
class StepSpec:
    """Sizes of a rank's share of a model."""
    d: int = 2048               # width of the residual stream
    hidden: int = 4096          # width between the two products of an expert
    experts: int = 8            # of this rank
    layers: int = 2
    vocab: int = 32000
    scale: float = 0.9          # of the residual stream
    eps: float = 1e-6
    seed: int = 0


def even_load(rows: int, experts: int) -> List[int]:
    """The rows of each expert when routing spreads them evenly."""
    return [rows * (e + 1) // experts - rows * e // experts for e in range(experts)]


class RankStep:
    """The weights of one rank on one GPU, and its step."""

    def __init__(self, spec: StepSpec = StepSpec(), dtype=torch.bfloat16, device: str = "cuda:0"):
        self.spec, self.dtype, self.device = spec, dtype, torch.device(device)
        g = torch.Generator(device=self.device).manual_seed(spec.seed)

        def normal(*shape, std, mean=0.0):
            t = torch.empty(shape, dtype=dtype, device=self.device).normal_(mean, std, generator=g)
            return t.requires_grad_()
        s = spec
        self.layers = [dict(up=normal(s.experts, s.hidden, s.d, std=s.d ** -0.5), down=normal(s.experts, s.d, s.hidden, std=s.hidden ** -0.5),
                            gate=normal(1, s.d, std=0.1, mean=1.0), post=normal(s.d, std=0.1, mean=1.0), pre=normal(s.d, std=0.1, mean=1.0))
                       for _ in range(s.layers)]
        self.vocabulary = normal(s.vocab, s.d, std=s.d ** -0.5)

    def weights(self) -> List[torch.Tensor]:
        return [w for layer in self.layers for w in layer.values()] + [self.vocabulary]

    def batch(self, load: Sequence[int], seed: int = 0, masked: float = 0.0):
        """Rows sorted by expert, as many as `load` says for each, and their labels: (h [rows, d], offsets, labels)."""
        if len(load) != self.spec.experts or min(load) < 0:
            raise ValueError(f"a load of {len(load)} experts, the step has {self.spec.experts}")
        g = torch.Generator(device=self.device).manual_seed(seed)
        rows = int(sum(load))
        h = torch.empty(rows, self.spec.d, dtype=self.dtype, device=self.device).normal_(generator=g)
        offsets = torch.tensor(np.concatenate([[0], np.cumsum(load)]), dtype=torch.int32, device=self.device)
        labels = torch.randint(0, self.spec.vocab, (rows,), generator=g, device=self.device)
        labels[torch.rand(rows, generator=g, device=self.device) < masked] = -1
        return h, offsets, labels

    def loss(self, h, offsets, labels) -> torch.Tensor:
        """The mean loss of the rows that have a target."""
        u = h
        for w in self.layers:
            inner = torch.nn.functional.silu(step.ExpertProduct.apply(u, w["up"], offsets))
            block = step.ExpertProduct.apply(inner, w["down"], offsets)
            h, u = step.NormResidual.apply(h, block, w["gate"], w["post"], w["pre"], self.spec.scale, self.spec.eps)
        loss = step.VocabLoss.apply(u, self.vocabulary, labels)
        return loss.sum() / ((labels >= 0) & (labels < self.spec.vocab)).sum().clamp(min=1)

    def gradients(self, h, offsets, labels):
        """One step: (loss, gradients of weights())."""
        loss = self.loss(h, offsets, labels)
        return loss.detach(), torch.autograd.grad(loss, self.weights())

    def measure(self, loads: Sequence[Sequence[int]], repeats: int = 5) -> np.ndarray:
        """Nanoseconds that a step takes with each of the loads: the median of `repeats`, after one that does not count."""
        out = []
        with torch.cuda.device(self.device):
            for i, load in enumerate(loads):
                batch = self.batch(load, seed=i)
                times = []
                for k in range(repeats + 1):
                    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                    begin.record()
                    self.gradients(*batch)
                    end.record()
                    end.synchronize()
                    if k:
                        times.append(begin.elapsed_time(end))
                out.append(int(np.median(times) * 1e6))
        return np.asarray(out, dtype=np.int64)


def trace(compute_ns: np.ndarray, n_slots: int = 200, seed: int = 0) -> tg.Trace:
    """The records of a job of one ring, as many ranks as there are times: rank r computes for compute_ns[r] between two collectives.  (The
    generator's faults are left out: what is uneven is the computation.)"""
    compute_ns = np.asarray(compute_ns, dtype=np.int64)
    spec = tg.config1(n_slots=n_slots, seed=seed, faults=False)
    spec = replace(spec, layout=tg.Layout3D(tp=len(compute_ns), pp=1, dp=1))
    return tg.propagate(tg.generate(spec), compute_ns)


def main(argv=None) -> int:
    p = argparse.ArgumentParser(description="Times a training step's computation on this card for an ordinary and for a larger load, has the analyzer name "
                                            "the late rank in the trace of a job made of these times, and compares a rank's time with its load's.")
    p.add_argument("--ranks", type=int, default=16)
    p.add_argument("--rows", type=int, default=4096, help="rows of a rank")
    p.add_argument("--busy-rank", type=int, default=5, help="the rank that routing sends more rows")
    p.add_argument("--times", type=float, default=2.0, help="how many times the rows of the others")
    p.add_argument("--slots", type=int, default=200, help="collectives of the trace")
    p.add_argument("--took-us", type=float, help="what the busy rank's step took in its job, on its own card")
    a = p.parse_args(argv)
    if a.ranks < 3 or not 0 <= a.busy_rank < a.ranks or a.rows < 1:
        p.error("at least 3 ranks, one of them busy, and a row")
    if a.took_us is not None and not a.took_us > 0:
        p.error("a step takes more than no time")
    from . import ccld
    work = RankStep()
    usual, busy = even_load(a.rows, work.spec.experts), even_load(int(a.rows * a.times), work.spec.experts)
    usual_ns, busy_ns = work.measure([usual, busy])
    compute_ns = np.full(a.ranks, usual_ns, dtype=np.int64)
    compute_ns[a.busy_rank] = busy_ns
    tr = trace(compute_ns, n_slots=a.slots)
    # flagged: entries that are late by a fifth of a step and more
    an = ccld.Analyzer(tr.topo, max_window_records=tr.n, lag_floor_ns=max(int(usual_ns) // 5, 50_000))
    an.ingest(an.to_device(tr.cols))
    result = an.analyze_window(int(tr.cols["t_exit"].max()) + 1, n_records=tr.n)
    blame, order = an.rank_blame()
    an.close()
    print(f"a step of {sum(usual)} rows: {usual_ns / 1e3:.0f} us, of {sum(busy)} rows: {busy_ns / 1e3:.0f} us "
          f"({usual_ns / sum(usual):.0f} and {busy_ns / sum(busy):.0f} ns a row)")
    named = int(order[0])
    print(f"{result.n_records} records, {result.n_flag} flags; most late entries: rank {named} ({int(blame['n_late_enter'][named])} of {a.slots})")
    print(f"its rows take {busy_ns / usual_ns:.2f} times as long as the others' on this card" +
          (f"; it took {a.took_us * 1e3 / busy_ns:.2f} times as long as its rows take here" if a.took_us else ""))
    return 0 if named == a.busy_rank else 1


if __name__ == "__main__":
    raise SystemExit(main())
