"""What the command says of a rank's time, and a step in half precision, whose roundings are an eighth of bfloat16's."""
import re

import pytest
import torch

from paper_2605_04478_amd import rankstep
from tests.test_gpu_rankstep import SPEC, _in_64_bits

pytestmark = pytest.mark.gpu
JOB = ["--ranks", "6", "--busy-rank", "4", "--rows", "2048", "--times", "4", "--slots", "30"]


def test_the_command_compares_a_ranks_time_with_its_loads(capsys):
    """Both loads are timed on this card: they say nothing of the rank's own card, unless the time that it took there is given."""
    assert rankstep.main(JOB) == 0
    said = capsys.readouterr().out
    assert "card is as fast" not in said and "it took" not in said
    assert rankstep.main(JOB + ["--took-us", "1000000"]) == 0
    said = capsys.readouterr().out
    busy_us = float(re.search(r"of 8192 rows: (\d+) us", said).group(1))
    times = float(re.search(r"it took ([\d.]+) times as long as its rows take here", said).group(1))
    assert abs(times - 1e6 / busy_us) <= 0.01 + times / busy_us          # both are rounded
    with pytest.raises(SystemExit):
        rankstep.main(JOB + ["--took-us", "-1"])


@pytest.mark.parametrize("load,masked", [((30, 0, 50, 17), 0.3), ((1, 1, 1, 1), 0.0), ((60, 50, 0, 0), 0.5)], ids=str)
def test_half_precision_step_against_64_bits(load, masked):
    work = rankstep.RankStep(SPEC, dtype=torch.float16)
    batch = work.batch(load, seed=3, masked=masked)
    loss, grads = work.gradients(*batch)
    want_loss, want = _in_64_bits(work, *batch)
    # 25 roundings of half a step of 2^-10, as counted for bfloat16, and as many of half a step of the subnormal numbers, 2^-24
    bound, least = 25 * 2.0 ** -11, 25 * 2.0 ** -25
    assert abs(float(loss) - float(want_loss)) <= bound * max(1.0, abs(float(want_loss)))
    for w, g, x in zip(work.weights(), grads, want):
        assert g.shape == w.shape and g.dtype == w.dtype
        assert float((g.double().cpu() - x).norm()) <= bound * float(x.norm()) + least * x.numel() ** 0.5, tuple(w.shape)
