"""Log probabilities and distillation in each form that rows and vocabulary choose: the forms for many rows that only large calls reach."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1805_10387_amd as mp
from gpu_util import *
import test_gpu_token_logprobs as T


def test_more_rows_than_the_longest_forms_launch_could_count():
    """2^23 + 5 short rows, each with 64 lanes: the rows of a smaller call over and over, bit by bit."""
    rows, vocab, ld, few = (1 << 23) + 5, 3, 8, 1021
    x = T.rows_of("ties", few, ld).astype(np.float16)
    which = torch.arange(rows, device="cuda") % few
    small, t = torch.from_numpy(x).cuda(), i32(np.arange(few) % 4 - 1)
    big, targets = small[which], t[which]

    def run(n, logits, t):
        out = [empty32(n) for _ in range(3)] + [torch.empty(n, 2, dtype=torch.int32, device="cuda"), empty32(n, 2)]
        mp.mp_token_logprobs(n, vocab, 2, logits, ld, t, 1.0, *out)
        return out

    for a, b in zip(run(few, small, t), run(rows, big, targets)):
        assert torch.equal(a[which], b)
