"""GPU: the cut of rows whose weight falls on the border of top-p's share.

a tokens of logit 0 and b of logit z < 0, the others masked, top-k above a + b,
top-p 1/2, such that half of the weight is that of the first a + m tokens to
within the rounding of a 64-bit sum (found by a search over z and T): a sum
whose order depends on the waves' timing takes m or m + 1 of the lighter ones
by chance.  Equal rows have to give equal results, within a call and from one
call to the next."""
import numpy as np
import pytest
import torch

from paper_2609_26638_amd import dvs

pytestmark = pytest.mark.gpu

#        a    b    m    z                     T
CASES = [(181, 598, 149, -0.6054705381393433, 1.1982742547988892),
         (96, 594, 245, -0.09439188987016678, 1.1792690753936768),
         (196, 482, 125, -0.24236547946929932, 1.437324047088623),
         (187, 374, 93, -0.003952059894800186, 0.7410094738006592),
         (65, 470, 193, -0.18099185824394226, 0.7058151960372925),
         (91, 440, 173, -0.026257360354065895, 0.8095309734344482),
         (91, 576, 75, -1.3798428773880005, 0.8939238786697388),
         (192, 370, 87, -0.020899532362818718, 1.0135914087295532),
         (104, 413, 99, -1.3546000719070435, 1.8652054071426392),
         (182, 341, 79, -0.00798806268721819, 1.457817792892456),
         (67, 409, 170, -0.04101415351033211, 1.3943806886672974),
         (101, 509, 130, -1.6366571187973022, 1.8138073682785034),
         (118, 598, 206, -0.5900036096572876, 1.2965344190597534),
         (142, 560, 205, -0.02772694267332554, 0.5058900713920593)]


@pytest.mark.parametrize("rows", [200, 400])
@pytest.mark.parametrize("a,b,m,z,T", CASES)
def test_equal_rows_are_cut_alike(a, b, m, z, T, rows):
    V = 3001
    at = np.random.default_rng([a, b]).permutation(V)
    row = np.full(V, -np.inf, np.float32)
    row[at[:a]], row[at[a:a + b]] = 0.0, z
    zt = torch.from_numpy(row).cuda().expand(rows, V).contiguous()
    f = lambda x: torch.full((rows,), x, device="cuda")   # noqa: E731
    seen = set()
    for _ in range(8):
        tok, prob = dvs.sample_filtered(zt, f(0.875), f(T), f(1000).int(), f(0.5))
        seen |= set(zip(tok.tolist(), prob.view(torch.int32).tolist()))
    assert len(seen) == 1, sorted(seen)
