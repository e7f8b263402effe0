"""The fusion scorer's operators on the GPU where they were once wrong, each against a 64-bit form
or against the same call made again."""

import numpy as np
import pytest
import torch

import paper_2603_14002_amd as lbm
from tests import scorer_ref as ref
from tests.gpu_util import say
from tests.test_gpu_scorer import DT, close, dev, handles, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a ROCm device")
    lbm.lib()


# ------------------------------------------------------------------ attention in bf16

BF16 = [  # new, length, page, q heads, kv heads, D, window: each of the kernels, and the parts' join
    ([1, 3], [200, 40], 16, 8, 2, 64, 0),
    ([1], [1500], 64, 4, 1, 128, 0),
    ([2], [400], 32, 2, 1, 256, 90),
    ([1] * 530, [1 + i % 40 for i in range(530)], 16, 4, 4, 64, 0),
    ([650], [700], 16, 128, 8, 64, 0),
    ([310, 300], [330, 333], 64, 128, 4, 128, 90),
    ([305], [306], 128, 256, 2, 256, 0),
]


@pytest.mark.parametrize("case", range(len(BF16)))
def test_attend_bf16_rounds_the_output_alone(case):
    """With bf16 activations an output is off by its own rounding to bf16, and beside that by no more than 2^-16 of
    the probabilities (two pieces of 8 significant bits) and the 32-bit sums' errors."""
    new, length, P, Hq, H, D, window = BF16[case]
    say(f"[case] attend bf16 {case}")
    rng = np.random.default_rng(500 + case)
    R = ref.Ragged(new, length, P, H, D, seed=case)
    for s, n in enumerate(length):
        R.put(s, randn(rng, n, H, D, dtype=torch.float64) + 2 * randn(rng, 1, H, D, dtype=torch.float64), randn(rng, n, H, D, dtype=torch.float64))
    q = dev(randn(rng, R.n_rows, Hq, D, dtype=torch.bfloat16))
    cache, batch = handles(R)
    out, _ = lbm.lb_kv_attend(cache, batch, q, D ** -0.5, window=window)
    m = 0
    for s, n in enumerate(new):
        if s < 4 or s % 40 == 0:
            k, v = R.get(s, length[s])
            want, _, mass, reach = ref.attend(q.cpu()[m:m + n].double(), k, v, D ** -0.5, length[s] - n, window)
            # scores summed in 32 bits over D channels move a probability by twice their error; the exponential's and
            # the sums' own roundings; the output's half step on top
            delta = (D + 8) * 2.0 ** -23 * reach + 2.0 ** -21 * (1 + reach)
            rest = (2.0 ** -16 + 4 * delta + length[s] * 2.0 ** -24).unsqueeze(-1) * mass
            close(out[m:m + n], want, ref.EPS[torch.bfloat16] * (want.abs() + rest) + rest, f"sequence {s}")
        m += n
