"""Rows shared by two, four and eight CTAs draw the same tokens, counts and log-probabilities, to the last bit, as rows of one CTA."""
import pytest
import torch

from paper_2605_14978_b200 import binding as B

from test_gpu_sample import TYPES, check, make

pytestmark = pytest.mark.gpu
FILTERS = [dict(), dict(top_p=0.95), dict(temperature=0.7, top_k=20, min_p=0.01), dict(temperature=400.0, top_k=50000, top_p=0.9)]


@pytest.mark.parametrize("dtype", TYPES)
def test_the_same_whichever_way_a_row_is_cut(dtype):
    R, V = 700, 70001                                        # 700 rows: a CTA each; 8751 units and more to cut
    z, u = make(R, V, dtype, seed=14)
    z[1::10] = z[1::10] * 3000.0                             # searched, of 16-bit rows too
    z[2::10] = (z[2::10] * 4.0).round()                      # many equal ones
    z[3::10, : V // 2] = -float("inf")
    z[4::10, 50:] = -float("inf")
    z[5::10] = 0.5                                           # more equal ones than a count holds
    for k in FILTERS:
        whole = B.sample_tokens(z, u, **k)
        check(z[:10], u[:10], {n: t[:10] for n, t in whole.items()}, **k)
        for rows in (1, 7, 10, 30, 60, 120):                 # eight CTAs to a row, four, two
            for start in (0, 5, R - rows):
                part = slice(start, start + rows)
                few = B.sample_tokens(z[part], u[part], **k)
                assert all(torch.equal(few[n].view(torch.int32), whole[n][part].view(torch.int32)) for n in few), (rows, start, k)
    torch.cuda.synchronize()
