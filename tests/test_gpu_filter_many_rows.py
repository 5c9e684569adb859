"""GPU: more rows than one launch takes (2^21 workgroups): the rows around the
launches' borders and at the ends give what calls of these rows alone give."""
import pytest
import torch

from paper_2609_26638_amd import dvs

pytestmark = pytest.mark.gpu

LAUNCH = 1 << 21


def _ends(n):
    return [slice(0, 300), slice(n - 300, n)] + [slice(b - 150, b + 150)
                                                 for b in range(LAUNCH, n - 150, LAUNCH)]


def test_sampler():
    rows, V = (1 << 23) + 1001, 3              # at 512 threads a row: more than 2^32
    gen = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn((rows, V), device="cuda", generator=gen).bfloat16()
    u = torch.rand(rows, device="cuda", generator=gen)
    p = torch.rand(rows, device="cuda", generator=gen)
    out = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    prob = torch.full((rows,), -1.0, device="cuda")
    dvs.sample_filtered(z, u, top_p=p, token_out=out, prob_out=prob)
    assert int(out.min()) == 0 and int(out.max()) == V - 1 and float(prob.min()) > 0
    for s in _ends(rows):
        tok, pr = dvs.sample_filtered(z[s], u[s], top_p=p[s])
        assert torch.equal(out[s], tok) and torch.equal(prob[s], pr)


def test_acceptance():
    S, B, V = LAUNCH + 1001, 2, 2              # 5 rows a sequence
    gen = torch.Generator(device="cuda").manual_seed(2)
    zv = torch.randn((S, B + 1, V), device="cuda", generator=gen)
    zd = torch.randn((S, B, V), device="cuda", generator=gen)
    draft = torch.randint(0, V, (S, B), device="cuda", generator=gen, dtype=torch.int32)
    u = torch.rand((S, B + 1), device="cuda", generator=gen)
    A, tok = (torch.full((S,), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    dvs.accept_sampled(zv, zd, draft, u, accept_len=A, token_out=tok)
    assert int(A.min()) == 0 and int(A.max()) == B and int(tok.min()) == 0 and int(tok.max()) == 1
    for s in _ends(S):
        a, t = dvs.accept_sampled(zv[s], zd[s], draft[s], u[s])
        assert torch.equal(A[s], a) and torch.equal(tok[s], t)
