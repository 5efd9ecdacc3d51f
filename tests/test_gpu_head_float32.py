"""The head's log-probabilities against those from a float32 product of the same inputs: both against float64, as norms over the rows.
What the tensor cores' additions cut off must not show: no more than twice the float32 product's error, or 1e-6."""
import numpy as np
import pytest
import torch

from paper_2605_14978_b200 import binding as B

import test_gpu_head as head

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("temperature", [1.0, 0.7])
@pytest.mark.parametrize("D", [264, 520, 1024, 2048, 4096])
@pytest.mark.parametrize("T", [20, 100, 300])
def test_as_exact_as_a_float32_product(T, D, temperature, dtype):
    temperature, err = float(np.float32(temperature)), np.zeros((2, 2))
    for seed in range(3):
        h, w, tok, _ = head.make(T, 8000, D, dtype, seed=80 + seed, masked=0.0)
        y = tok.long()[:, None]
        z = h.double() @ w.double().t() / temperature
        want = (torch.log_softmax(z, 1).gather(1, y)[:, 0], torch.logsumexp(z, 1))
        out = B.head_logprob(h, w, tok, temperature=temperature)
        z = (h.float() @ w.float().t()).double() / temperature
        plain = (torch.log_softmax(z, 1).gather(1, y)[:, 0].float(), torch.logsumexp(z, 1).float())
        for i, got in enumerate(((out["logp"], out["lse"]), plain)):
            for k in range(2):
                err[i, k] += float((got[k].double() - want[k]).square().sum() / want[k].square().sum()) / 3
    own, product = np.sqrt(err)
    assert (own <= np.maximum(2 * product, 1e-6)).all(), (own, product)
