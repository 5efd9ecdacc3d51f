"""How exact the masses of a searched row are: draws next to a border of millions of equal weights, where each weight's rounding counts as often
as the weight."""
import numpy as np
import pytest
import torch

from paper_2605_14978_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
V, ROWS = 1 << 22, 5


def near_borders(z1, z2):
    """Rows (where the lower logits start, uniform, token) whose draw falls on one of the lower half's equal weights, close to the border of two.

    Logits: a zero, z1 up to the start, z2 from there on.  With A the mass before the start, M and w the number and the weight behind it,
    the draw falls on place floor(x) from the start, x = u M - (1 - u) A / w.  Weights off by d of themselves move x by up to
    (1 - u) A / w * 2 d."""
    e1, e2 = np.exp(-np.longdouble(z2)), np.exp(np.longdouble(z1) - np.longdouble(z2))       # 64 bits of mantissa: x is right to 1e-12
    rows, start = [], V // 2
    while len(rows) < ROWS:
        start -= 1009
        M, a_w = V - start, e1 + (start - 1) * e2
        lo = int(np.ceil(float(a_w / (a_w + M)) * 2 ** 24)) + 1
        u = np.arange(lo, min(lo + (1 << 20), 1 << 24)).astype(np.longdouble) / 2 ** 24
        x = u * M - (1 - u) * a_w
        gap = np.abs(x - np.rint(x))
        # what weights right to 6e-14 of themselves allow, and 2e-14 for float64's share in them; no more than eight times as much
        bound = (1 - u) * a_w * 2 * 8e-14 + M * 1e-15
        at = np.flatnonzero((gap > bound) & (gap < 8 * bound))
        if len(at):
            rows.append((start, np.float32(u[at[0]]), start + int(np.floor(x[at[0]]))))
    return rows


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("z1,z2", [(-0.75, -2.75), (-1.25, -3.5), (-0.3125, -1.0), (-2.5, -3.25)])
def test_draws_next_to_the_border_of_equal_weights(z1, z2, dtype):
    rows = near_borders(z1, z2)
    z = torch.full((ROWS, V), z1, dtype=dtype, device=DEV)
    z[:, 0] = 0.0
    for i, (start, _, _) in enumerate(rows):
        z[i, start:] = z2
    got = B.sample_tokens(z, torch.tensor([float(u) for _, u, _ in rows], device=DEV))
    torch.cuda.synchronize()
    np.testing.assert_array_equal(got["tokens"].cpu().numpy(), [t for _, _, t in rows])
    assert torch.all(got["kept"] == V)
