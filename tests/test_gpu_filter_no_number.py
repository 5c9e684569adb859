"""GPU: rows without a value above -inf (masked tokens and NaN alone).  They give
the rule of argmax_accept, the lowest index of -inf, 0 when every value is NaN,
with probability 0 and the error bit, in the sampler and in the acceptance."""
import numpy as np
import pytest
import torch

from oracle import filter as of
from paper_2609_26638_amd import dvs

pytestmark = pytest.mark.gpu

SIZES = [1, 2, 3, 5, 9, 300, 301, 1003, 1021, 32003, 65543]


def _rows(V):
    """NaN alone; all masked; one masked token, at either end, in the middle and
    behind the last whole vectors; NaN behind masked ones."""
    z = [np.full(V, np.nan), np.full(V, -np.inf)]
    for i in sorted({0, V // 2, V // 8 * 8, V // 4 * 4, V - 1}):
        r = np.full(V, np.nan)
        r[min(i, V - 1)] = -np.inf
        z.append(r)
    r = np.full(V, -np.inf)
    r[:V // 2] = np.nan
    return np.array(z + [r])


def _dev(z, dtype):
    t = torch.from_numpy(np.asarray(z, np.float32))
    return (t.to(torch.bfloat16) if dtype == "bf16" else t).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", SIZES)
def test_sampler(V, dtype):
    z = _rows(V)
    want = [of.no_number(r) for r in z]
    for rows in (len(z), 300):                     # a CU to every row, and more rows than CUs
        at = np.arange(rows) % len(z)
        zt, n = _dev(z, dtype)[torch.from_numpy(at).cuda()], rows
        u = torch.rand(n, device="cuda", generator=torch.Generator("cuda").manual_seed(V))
        for par in ({}, dict(temperature=torch.zeros(n, device="cuda")),
                    dict(top_p=torch.full((n,), 0.9, device="cuda"),
                         top_k=torch.full((n,), 7, dtype=torch.int32, device="cuda"))):
            err = torch.zeros(1, dtype=torch.int32, device="cuda")
            tok, prob = dvs.sample_filtered(zt, u, err=err, **par)
            assert tok.tolist() == [want[i] for i in at]
            assert not prob.any() and int(err.item()) == dvs.ERR_NONFINITE


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", SIZES)
def test_acceptance(V, dtype):
    """The first verify row of each sequence has no number, so that its draft is
    refused; or the second, whose draft row has none either."""
    z = _rows(V)
    n = len(z)
    rng = np.random.default_rng(V)
    for S in (2 * n, 120) if V < 2000 else (2 * n,):   # 5 rows each
        zv, zd = rng.standard_normal((S, 3, V)), rng.standard_normal((S, 2, V))
        zv, zd = np.float32(zv), np.float32(zd)
        if dtype == "bf16":
            r = lambda a: torch.from_numpy(a).bfloat16().float().numpy()   # noqa: E731
            zv, zd = r(zv), r(zd)
        draft = np.zeros((S, 2), np.int32)
        u = rng.random((S, 3)).astype(np.float32)
        want = []
        for s in range(S):
            if s % 2:
                zv[s, 1] = zd[s, 1] = z[s // 2 % n]
                zd[s, 0], u[s, 0] = zv[s, 0], 0.5  # the first draft is accepted
            else:
                zv[s, 0] = z[s // 2 % n]
            p, q = ([of.probs(of.kept_weights(r)) for r in a[s]] for a in (zv, zd))
            want.append(of.accept(np.array(p), np.array(q), draft[s], u[s].astype(np.float64), zv[s]))
            assert want[-1] == (s % 2, of.no_number(z[s // 2 % n]))
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        A, tok = dvs.accept_sampled(_dev(zv, dtype), _dev(zd, dtype), torch.from_numpy(draft).cuda(),
                                    torch.from_numpy(u).cuda(), err=err)
        assert list(zip(A.tolist(), tok.tolist())) == want
        assert int(err.item()) == dvs.ERR_NONFINITE


def test_draft_rows_without_a_number_weigh_nothing():
    """q = 0: the draft is accepted where p keeps it."""
    S, V = 6, 301
    zv = np.float32(np.random.default_rng(1).standard_normal((S, 2, V)))
    zd = np.full((S, 1, V), np.nan)
    zd[:, :, V - 1] = -np.inf
    A, tok = dvs.accept_sampled(_dev(zv, "f32"), _dev(zd, "f32"),
                                torch.arange(S, dtype=torch.int32, device="cuda").view(S, 1),
                                torch.full((S, 2), 0.5, device="cuda"))
    assert A.tolist() == [1] * S
    assert tok.tolist() == [of.sample(zv[s, 1], 0.5)[0] for s in range(S)]
