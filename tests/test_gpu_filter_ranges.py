"""GPU: sample_filtered at the ends of its ranges, against the float64 oracle:
top-k of thousands of distinct logits, vocabularies up to 2^22, and shares of
top-p so close to 1 that the cut falls among tokens of 1e-12 of the weight.

What the two sides may differ by: the kernel's weights are off by 4e-14 of
themselves, and a thread that adds up to 4096 of them to a sum of 1 rounds each
time, by 1.1e-16 at most, 4e-15 in all on the average.  The oracle's cut and
draw are exact to 2^-64.  So a cut or a draw among light tokens has to lie
further than 1e-14 of the whole from the sums next to it, which every row is
looked over for on the host before its result."""
import numpy as np
import pytest
import torch

from oracle import filter as of
from paper_2609_26638_amd import dvs

pytestmark = pytest.mark.gpu

PROB_TOL = 2.0 ** -24 * (1 + 1e-3) + 1e-9


def _check(z, par, dtype="f32"):
    """par: u, T, k, p, m, one entry a row."""
    t = torch.from_numpy(np.asarray(z, np.float32))
    t = t.bfloat16() if dtype == "bf16" else t
    z64 = t.double().numpy()
    d = {n: torch.from_numpy(np.asarray(a, np.int32 if n == "k" else np.float32)).cuda()
         for n, a in par.items()}
    tok, prob = dvs.sample_filtered(t.cuda(), d["u"], d["T"], d["k"], d["p"], d["m"])
    tok, prob = tok.tolist(), prob.tolist()
    f32 = {n: np.asarray(a, np.int32 if n == "k" else np.float32) for n, a in par.items()}
    for r in range(len(z64)):
        u, T, k, p, m = (f32[n][r].item() for n in ("u", "T", "k", "p", "m"))
        want, pr = of.sample(z64[r], u, T, k, p, m)
        what = f"row {r}: u {u} T {T} k {k} p {p} m {m}"
        assert tok[r] == want, f"{what}: token {tok[r]}, oracle {want}"
        assert abs(prob[r] - pr) <= PROB_TOL * pr, f"{what}: {prob[r]}, oracle {pr}"


def _cycle(rows, *values):
    return [values[i % len(values)] for i in range(rows)]


@pytest.mark.parametrize("dtype,V,rows", [("f32", 65536, 48), ("f32", 40009, 270),
                                          ("bf16", 65536, 24)])
def test_top_k_of_thousands(V, rows, dtype):
    """More than a thread's parts tell, more than a list holds, all but one."""
    rng = np.random.default_rng([V, rows])
    z = rng.standard_normal((rows, V)) * rng.choice([0.3, 1.5, 4.0], (rows, 1))
    z[3::8, rng.random(V) < 0.5] = -np.inf
    _check(z, dict(u=rng.random(rows), T=rng.uniform(0.5, 1.5, rows),
                   k=_cycle(rows, 4097, 9000, 20000, V - 1, 3000, 8193, 16385),
                   p=_cycle(rows, 1.0, 0.9, 0.999, 1.0, 0.5), m=_cycle(rows, 0.0, 0.0, 1e-3)), dtype)


@pytest.mark.parametrize("V", [1 << 20, (1 << 22) - 3, 1 << 22])
@pytest.mark.parametrize("sigma", [0.05, 1.0, 4.0])
def test_largest_vocabularies(V, sigma):
    rows = 6
    rng = np.random.default_rng([V, int(sigma * 100)])
    z = rng.standard_normal((rows, V), dtype=np.float32) * np.float32(sigma)
    _check(z, dict(u=rng.random(rows), T=[1.0, 0.7, 1.0, 1.2, 1.0, 0.9],
                   k=[0, 0, 50, 0, V // 3, 0], p=[1.0, 0.9, 1.0, 0.99, 0.9, 0.97],
                   m=[0.0, 0.0, 0.0, 0.0, 0.0, 0.02]))


def _margin(z, p, k, u):
    """Distance of top-p's border from the sums next to it, and of the draw's,
    as a share of the whole."""
    o = -np.sort(-z.astype(np.float64), kind="stable")[:k if k else None]
    c = np.cumsum(np.exp(o - o[0]).astype(np.longdouble))
    i = int(np.searchsorted(c, np.longdouble(p) * c[-1]))
    cut = min(abs(c[j] / c[-1] - np.longdouble(p)) for j in range(max(0, i - 1), min(i + 2, len(c))))
    w = of.kept_weights(z, 1.0, k, p)
    c = np.cumsum(w.astype(np.longdouble))
    t = np.longdouble(u) * c[-1]
    i = int(np.searchsorted(c, t, side="right"))
    return float(min(cut, abs(c[i] - t) / c[-1], abs(c[i - 1] - t) / c[-1] if i else 1.0))


@pytest.mark.parametrize("V,k,lo,hi,one_minus_p", [
    (1 << 22, 0, -27.6, -27.2, [2e-6, 1e-6, 4e-6]),       # 4 M tokens of 2^-39.5 each
    (1 << 20, 0, -27.0, -20.0, [1e-5, 1e-6, 1e-4]),
    (1 << 20, 700000, -27.6, -27.2, [4e-7, 6e-7, 2e-7]),  # top-k, then top-p of these
    (1 << 20, 10000, -27.0, -24.0, [1e-7, 3e-8, 6e-8]),
    (70001, 0, -30.0, -22.0, [1e-6, 1e-7, 1e-5])])
def test_cuts_among_the_lightest(V, k, lo, hi, one_minus_p):
    """One heavy token and a tail of light ones: the share that top-p leaves out is
    a part of the tail, and so is what u close to 1 draws."""
    rows = 3
    rng = np.random.default_rng([V, k])
    z = rng.uniform(lo, hi, (rows, V)).astype(np.float32)
    z[:, 12345] = 0.0
    p = np.float32(1 - np.array(one_minus_p))
    u = np.float32([0.5, 1 - 2.0 ** -23, 1 - 2.0 ** -24])
    margins = [_margin(z[r].astype(np.float64), float(p[r]), k, float(u[r])) for r in range(rows)]
    print("margins", margins)
    assert min(margins) > 1e-14
    _check(z, dict(u=u, T=np.ones(rows), k=[k] * rows, p=p, m=np.zeros(rows)))
