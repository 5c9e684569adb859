"""GPU: sample_filtered and accept_sampled against the float64 oracle
(oracle/filter.py) on the same logits and uniforms.

Tokens and accepted lengths have to be equal.  Both sides take their
decisions on 64-bit weights; the kernel's running sums differ from the
oracle's by at most about 1e-11 of a row's weight (its cut is found on
fixed-point weights, 2^-45 of the largest each, 65536 of them), so that a
draw or a cut falls between the two once in some 10^6 rows.  Probabilities
are one rounding to fp32 of such a number: half a step, 2^-24, and 1e-9 for
the weights."""
import numpy as np
import pytest
import torch

from oracle import filter as of
from paper_2609_26638_amd import dvs

pytestmark = pytest.mark.gpu

PROB_TOL = 2.0 ** -24 * (1 + 1e-3) + 1e-9


def _rounded(z, dtype):
    t = torch.from_numpy(np.asarray(z, np.float32))
    t = t.to(torch.bfloat16) if dtype == "bf16" else t
    return t.cuda(), t.double().numpy()


def _params(rows):
    """Every combination of edge values and ordinary ones, cycled over rows."""
    T = [0.7, 1.0, 0.0, 1.3, 1e-6, 1e4, np.inf, 0.5, -1.0, np.nan]
    k = [0, 5, 1, 50, 2, -3, 1 << 30, 300, 0, 2000]
    p = [1.0, 0.9, 0.5, 0.95, 0.0, 1e-9, 1 - 2.0 ** -24, 2.0, np.nan, 0.3, 0.99]
    m = [0.0, 0.05, 0.0, 1.0, 0.0, 1e-3, 2.0, -1.0, np.nan]
    u = [0.5, 0.0, 0.123456, 1 - 2.0 ** -24, 0.9, 0.3, 1.0, np.nan, 0.77, -1.0, 0.05, 0.61, 0.999]
    c = lambda a: np.array([a[i % len(a)] for i in range(rows)], np.float32)   # noqa: E731
    return dict(T=c(T), k=c(k).astype(np.int64).clip(-9, 2 ** 30).astype(np.int32), p=c(p), m=c(m),
                u=c(u))


def _logits(kind, rows, V, rng):
    z = rng.standard_normal((rows, V)) * 4
    if kind == "flat":
        z = rng.standard_normal((rows, V)) * 0.3
    elif kind == "equal":
        z = np.full((rows, V), 1.5)
    elif kind == "levels":
        z = rng.integers(-2, 3, (rows, V)) * 1.0
        z[z == 0] *= np.where(rng.random(np.sum(z == 0)) < 0.5, -1, 1)    # -0 and +0
    elif kind == "masked":
        z[rng.random((rows, V)) < 0.9] = -np.inf
        z[::3] = np.where(rng.random((len(z[::3]), V)) < 0.5, -3.3895e38, z[::3])
        z[1::7] = -np.inf                                                  # nothing left
        z[2::7] = -np.inf
        z[2::7, V - 1] = -5.0                                              # a single token
    elif kind == "spread":
        z = np.sign(z) * 10.0 ** rng.uniform(-30, 30, (rows, V))
    return z


def _check(z64, par, got_t, got_p, group=1):
    for r in range(z64.shape[0]):
        g = r // group
        t, pr = of.sample(z64[r], float(par["u"][r]), float(par["T"][g]), int(par["k"][g]),
                          float(par["p"][g]), float(par["m"][g]))
        what = f"row {r}: " + ", ".join(f"{n} {par[n][g if n != 'u' else r]}" for n in par)
        assert int(got_t[r]) == t, f"{what}: token {int(got_t[r])}, oracle {t}"
        assert abs(float(got_p[r]) - pr) <= PROB_TOL * pr, f"{what}: {float(got_p[r])} {pr}"


def _dev(par):
    return {n: torch.from_numpy(np.ascontiguousarray(a)).cuda() for n, a in par.items()}


def _call(zt, d, **kw):
    return dvs.sample_filtered(zt, d["u"], d["T"], d["k"], d["p"], d["m"], **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["normal", "flat", "equal", "levels", "masked", "spread"])
@pytest.mark.parametrize("V", [1, 2, 3, 63, 64, 65, 255, 1000, 1024, 1025, 4097, 16389])
def test_sample_matches_oracle(V, kind, dtype):
    rows = 60
    rng = np.random.default_rng([V, len(kind), 3])
    zt, z64 = _rounded(_logits(kind, rows, V, rng), dtype)
    par = _params(rows)
    par["u"] = np.where(rng.random(rows) < 0.5, rng.random(rows), par["u"]).astype(np.float32)
    got_t, got_p = _call(zt, _dev(par))
    _check(z64, par, got_t.cpu().numpy(), got_p.cpu().numpy())


@pytest.mark.parametrize("dtype,kind,V", [("f32", "normal", 65536), ("bf16", "normal", 65536),
                                          ("bf16", "flat", 65536), ("f32", "masked", 65536),
                                          ("f32", "flat", 70001), ("bf16", "levels", 131072),
                                          ("f32", "normal", 150001)])
def test_large_vocabularies(dtype, kind, V):
    rows = 24
    rng = np.random.default_rng([V, 5])
    zt, z64 = _rounded(_logits(kind, rows, V, rng), dtype)
    par = _params(rows)
    par["T"] = rng.uniform(0.5, 1.5, rows).astype(np.float32)
    par["u"] = rng.random(rows).astype(np.float32)
    got_t, got_p = _call(zt, _dev(par))
    _check(z64, par, got_t.cpu().numpy(), got_p.cpu().numpy())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,kind", [(3, "levels"), (65, "masked"), (511, "flat"), (1025, "normal"),
                                    (4099, "equal"), (8192, "normal"), (20011, "flat"),
                                    (20011, "masked"), (9001, "spread"), (70001, "normal")])
def test_more_rows_than_the_chip_runs_at_once(V, kind, dtype):
    rows = 330
    rng = np.random.default_rng([V, len(kind), 7])
    zt, z64 = _rounded(_logits(kind, rows, V, rng), dtype)
    par = _params(rows)
    if kind in ("normal", "flat"):
        par["T"] = np.where(rng.random(rows) < 0.8, rng.uniform(0.3, 1.5, rows),
                            par["T"]).astype(np.float32)
    par["u"] = np.where(rng.random(rows) < 0.8, rng.random(rows), par["u"]).astype(np.float32)
    got_t, got_p = _call(zt, _dev(par))
    _check(z64, par, got_t.cpu().numpy(), got_p.cpu().numpy())


@pytest.mark.parametrize("dtype,V,rows,step", [("f32", 65536, 40, 0.0), ("bf16", 40007, 40, 0.0),
                                               ("f32", 17003, 40, 0.0), ("f32", 40007, 40, 0.25),
                                               ("f32", 65536, 40, 2.0), ("bf16", 20011, 300, 0.0),
                                               ("f32", 9007, 300, 0.5)])
def test_flat_rows_keep_more_than_a_list(V, rows, step, dtype):
    """Top-p over rows whose kept tokens are many thousands: cut by top-p, by
    min-p where it leaves less, by either; steps of equal logits; half masked."""
    rng = np.random.default_rng([V, rows, 17])
    z = rng.standard_normal((rows, V)) * rng.choice([0.1, 0.5, 1.0, 2.0], (rows, 1))
    if step:
        z = np.round(z / step) * step
    z[1::5][rng.random((len(z[1::5]), V)) < 0.5] = -np.inf
    zt, z64 = _rounded(z, dtype)
    c = lambda a: np.array([a[i % len(a)] for i in range(rows)], np.float32)   # noqa: E731
    par = dict(T=rng.choice([0.6, 1.0, 1.3, 50.0, 1e30], rows, p=[.3, .3, .2, .1, .1]).astype(np.float32),
               k=np.zeros(rows, np.int32), p=c([0.9, 0.5, 0.99, 0.7, 0.999, 0.95, 0.05]),
               m=c([0.0, 0.0, 0.02, 0.1, 0.0, 0.3, 1e-4, 0.9]), u=rng.random(rows).astype(np.float32))
    got_t, got_p = _call(zt, _dev(par))
    _check(z64, par, got_t.cpu().numpy(), got_p.cpu().numpy())


@pytest.mark.parametrize("offset", [-1e4, 1e3, 3e5])
@pytest.mark.parametrize("V,rows", [(257, 3000), (511, 3000), (4095, 600), (8193, 600)])
def test_logits_far_from_zero(V, rows, offset):
    """Their spacing is no longer small against T; shares close to 1."""
    rng = np.random.default_rng([V, int(abs(offset)), 29])
    z = rng.standard_normal((rows, V)) * rng.choice([0.05, 0.3, 1.0, 2.0], (rows, 1)) + offset
    zt, z64 = _rounded(z, "f32")
    par = dict(T=(10 ** rng.uniform(-2, 1, rows)).astype(np.float32), k=np.zeros(rows, np.int32),
               p=(1 - 10 ** rng.uniform(-4, -3, rows)).astype(np.float32),
               m=np.where(rng.random(rows) < 0.7, 0, 10 ** rng.uniform(-6, -3, rows)).astype(np.float32),
               u=rng.random(rows).astype(np.float32))
    got_t, got_p = _call(zt, _dev(par))
    _check(z64, par, got_t.cpu().numpy(), got_p.cpu().numpy())


@pytest.mark.parametrize("name", ["none", "k", "p", "m", "kp", "T"])
def test_each_filter_alone(name):
    rows, V = 16, 5003
    rng = np.random.default_rng(8)
    zt, z64 = _rounded(_logits("normal", rows, V, rng), "f32")
    par = dict(T=np.ones(rows, np.float32), k=np.zeros(rows, np.int32),
               p=np.ones(rows, np.float32), m=np.zeros(rows, np.float32),
               u=rng.random(rows).astype(np.float32))
    if "T" in name:
        par["T"] = rng.uniform(0.1, 3, rows).astype(np.float32)
    if "k" in name:
        par["k"] = rng.integers(1, 100, rows).astype(np.int32)
    if "p" in name:
        par["p"] = rng.random(rows).astype(np.float32)
    if "m" in name:
        par["m"] = (rng.random(rows) * 0.3).astype(np.float32)
    d = _dev(par)
    got_t, got_p = dvs.sample_filtered(zt, d["u"], d["T"] if "T" in name else None,
                                       d["k"] if "k" in name else None,
                                       d["p"] if "p" in name else None,
                                       d["m"] if "m" in name else None)
    _check(z64, par, got_t.cpu().numpy(), got_p.cpu().numpy())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("off,ld", [(0, 1024), (1, 1003), (3, 1500), (5, 1021)])
def test_rows_apart_and_unaligned(off, ld, dtype):
    """Rows inside a larger buffer that start on any element; what lies
    between them and around them is not read as logits."""
    rows, V = 20, 1003 if ld != 1024 else 1000
    rng = np.random.default_rng(ld)
    z = _logits("normal", rows, V, rng)
    buf = np.full(off + rows * ld + 64, np.nan, np.float32)
    flat, _ = _rounded(buf, dtype)
    view = flat[off:off + rows * ld].view(rows, ld)[:, :V]
    zt, z64 = _rounded(z, dtype)
    view.copy_(zt)
    par = _params(rows)
    d = _dev(par)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    got_t, got_p = _call(view, d, err=err)
    _check(z64, par, got_t.cpu().numpy(), got_p.cpu().numpy())
    assert int(err.item()) == 0


def test_grouped_parameters_and_leading_shape():
    S, R, V = 4, 6, 777
    rng = np.random.default_rng(2)
    zt, z64 = _rounded(_logits("normal", S * R, V, rng).reshape(S, R, V), "f32")
    par = _params(S)
    par["u"] = rng.random(S * R).astype(np.float32)
    d = _dev(par)
    d["u"] = d["u"].view(S, R)
    got_t, got_p = _call(zt, d)
    assert got_t.shape == (S, R) and got_p.shape == (S, R)
    _check(z64.reshape(S * R, V), par, got_t.cpu().numpy().ravel(), got_p.cpu().numpy().ravel(), R)


def test_non_finite_rows_flag_and_still_answer():
    V = 300
    z = np.random.default_rng(0).standard_normal((6, V))
    z[0, 7] = np.nan
    z[1, [9, 200]] = np.inf
    z[2] = np.nan
    z[3] = -np.inf
    z[3, 0] = np.nan
    z[4, 5] = -np.inf                        # a masked token: no error
    for rows, want in (([4, 5], 0), ([0], 4), ([1], 4), ([2], 4), ([3], 4), (range(6), 4)):
        zt, z64 = _rounded(z[list(rows)], "f32")
        par = _params(len(z64))
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        got_t, got_p = _call(zt, _dev(par), err=err)
        assert int(err.item()) == want
        _check(z64, par, got_t.cpu().numpy(), got_p.cpu().numpy())


def test_rows_do_not_depend_on_each_other_and_repeat():
    rows, V = 33, 9001
    rng = np.random.default_rng(4)
    zt, _ = _rounded(_logits("flat", rows, V, rng), "bf16")
    d = _dev(_params(rows))
    t, p = _call(zt, d)
    for _ in range(3):
        t2, p2 = _call(zt, d)
        assert torch.equal(t, t2) and torch.equal(p.view(torch.int32), p2.view(torch.int32))
    for r in (0, 17, 32):
        t1, p1 = _call(zt[r:r + 1], {n: a[r:r + 1] for n, a in d.items()})
        assert int(t1) == int(t[r]) and float(p1) == float(p[r])


def test_frequencies_follow_the_filtered_distribution():
    """An even grid of 4096 uniforms draws every token its probability's share
    of the grid, to one point per boundary."""
    N, V = 4096, 40
    z = np.random.default_rng(6).standard_normal(V) * 1.5
    zt, z64 = _rounded(np.tile(z, (N, 1)), "f32")
    u = ((np.arange(N) + 0.5) / N).astype(np.float32)
    one = np.ones(N, np.float32)
    d = _dev(dict(u=u, T=one * 0.8, k=np.full(N, 12, np.int32), p=one * 0.9, m=one * 0.02))
    t, _ = _call(zt, d)
    want = of.probs(of.kept_weights(z64[0], float(np.float32(0.8)), 12, float(np.float32(0.9)),
                                    float(np.float32(0.02))))
    got = np.bincount(t.cpu().numpy(), minlength=V) / N
    assert np.abs(got - want).max() <= 1.5 / N


# ---------------------------------------------------------------------------
# acceptance
# ---------------------------------------------------------------------------

def _accept_case(S, B, V, dtype, noise, seed):
    rng = np.random.default_rng(seed)
    zv = rng.standard_normal((S, B + 1, V)) * 2.5
    zd = zv[:, :B] + rng.standard_normal((S, B, V)) * noise
    par = _params(S)
    par["T"] = np.where(np.arange(S) % 5 == 4, 0.0, rng.uniform(0.5, 1.5, S)).astype(np.float32)
    zvt, zv64 = _rounded(zv, dtype)
    zdt, zd64 = _rounded(zd, dtype)
    u = rng.random((S, B + 1)).astype(np.float32)
    pp = lambda s: (float(par["T"][s]), int(par["k"][s]), float(par["p"][s]), float(par["m"][s]))  # noqa: E731
    pv = np.array([[of.probs(of.kept_weights(zv64[s, j], *pp(s))) for j in range(B + 1)]
                   for s in range(S)])
    qd = np.array([[of.probs(of.kept_weights(zd64[s, j], *pp(s))) for j in range(B)]
                   for s in range(S)])
    draft = np.array([[of.draw(qd[s, j], rng.random()) for j in range(B)] for s in range(S)],
                     np.int32)
    return zvt, zdt, par, u, pv, qd, draft


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S,B,V,noise", [(1, 1, 2, 0.5), (7, 3, 65, 0.3), (9, 16, 1021, 0.1),
                                         (5, 33, 300, 0.05), (3, 4, 32003, 0.2), (12, 2, 1, 0.1),
                                         (6, 8, 4096, 2.0)])
def test_accept_matches_oracle(S, B, V, noise, dtype):
    zvt, zdt, par, u, pv, qd, draft = _accept_case(S, B, V, dtype, noise, [S, B, V])
    if S > 2 and V > 2:
        draft[0, B - 1] = -1                 # no token
        draft[1, 0] = V                      # outside the vocabulary
        draft[2, 0] = int(np.argmin(pv[2, 0]))
    d = _dev(par)
    wide = torch.full((S, B + 3), -7, dtype=torch.int32, device="cuda")
    wide[:, :B] = torch.from_numpy(draft)
    A, tok = dvs.accept_sampled(zvt, zdt, wide, torch.from_numpy(u).cuda(), d["T"], d["k"], d["p"],
                                d["m"])
    A, tok = A.cpu().numpy(), tok.cpu().numpy()
    for s in range(S):
        want = of.accept(pv[s], qd[s], draft[s], u[s].astype(np.float64))
        assert (int(A[s]), int(tok[s])) == want, f"sequence {s}"


@pytest.mark.parametrize("sigma,p", [(0.3, 0.9), (1.0, 0.99), (2.5, 1.0)])
def test_accept_over_flat_rows(sigma, p):
    """More kept tokens than fit a list, in the draft rows and in the verify rows."""
    S, B, V = 3, 2, 20011
    rng = np.random.default_rng([S, V, 23])
    zv = rng.standard_normal((S, B + 1, V)) * sigma
    zd = zv[:, :B] + rng.standard_normal((S, B, V)) * 0.3
    zvt, zv64 = _rounded(zv, "f32")
    zdt, zd64 = _rounded(zd, "f32")
    pp = np.float32(p)
    pv = np.array([[of.probs(of.kept_weights(r, 1.0, 0, float(pp), 0.0)) for r in q] for q in zv64])
    qd = np.array([[of.probs(of.kept_weights(r, 1.0, 0, float(pp), 0.0)) for r in q] for q in zd64])
    draft = np.array([[of.draw(q, rng.random()) for q in row] for row in qd], np.int32)
    u = rng.random((S, B + 1)).astype(np.float32)
    u[0], u[1, :B], u[2, :B] = 0.999, 0.0, 0.5
    A, tok = dvs.accept_sampled(zvt, zdt, torch.from_numpy(draft).cuda(), torch.from_numpy(u).cuda(),
                                None, None, torch.full((S,), p, device="cuda"), None)
    for s in range(S):
        want = of.accept(pv[s], qd[s], draft[s], u[s].astype(np.float64))
        assert (int(A[s]), int(tok[s])) == want, f"sequence {s}"


def test_accept_takes_rows_inside_larger_tensors():
    """The draft rows of a round lie behind its boundary row, and rows may be
    padded."""
    S, B, V = 4, 5, 203
    zvt, zdt, par, u, pv, qd, draft = _accept_case(S, B, V, "f32", 0.2, 11)
    d = _dev(par)
    big_v = torch.full((S, B + 2, V + 9), float("nan"), device="cuda")
    big_d = torch.full((S, B + 1, V + 5), float("nan"), device="cuda")
    big_v[:, :B + 1, :V], big_d[:, 1:, :V] = zvt, zdt
    args = (torch.from_numpy(draft).cuda(), torch.from_numpy(u).cuda(), d["T"], d["k"], d["p"],
            d["m"])
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    A, tok = dvs.accept_sampled(zvt, zdt, *args)
    A2, tok2 = dvs.accept_sampled(big_v[:, :B + 1, :V], big_d[:, 1:, :V], *args, err=err)
    assert torch.equal(A, A2) and torch.equal(tok, tok2) and int(err.item()) == 0


def test_equal_rows_accept_every_draft():
    S, B, V = 6, 7, 900
    zvt, _, par, u, pv, _, _ = _accept_case(S, B, V, "f32", 0.0, 21)
    draft = np.array([[of.draw(pv[s, j], 0.37) for j in range(B)] for s in range(S)], np.int32)
    d = _dev(par)
    A, _ = dvs.accept_sampled(zvt, zvt[:, :B], torch.from_numpy(draft).cuda(),
                              torch.from_numpy(np.full_like(u, 1 - 2.0 ** -24)).cuda(), d["T"],
                              d["k"], d["p"], d["m"])
    assert A.tolist() == [B] * S


def test_capture_and_replay():
    """Both calls in one graph, replayed on changing inputs with eager work
    between, equal the eager calls."""
    S, B, V = 4, 3, 3001
    zvt, zdt, par, u, _, _, draft = _accept_case(S, B, V, "bf16", 0.3, 31)
    d = _dev(par)
    dr, ut = torch.from_numpy(draft).cuda(), torch.from_numpy(u).cuda()
    ws = dvs.Workspace(dvs.accept_workspace_bytes(S, B, V))
    out = [torch.zeros(S, dtype=torch.int32, device="cuda") for _ in range(3)]
    pr = torch.zeros(S, device="cuda")

    def step():
        dvs.accept_sampled(zvt, zdt, dr, ut, d["T"], d["k"], d["p"], d["m"], accept_len=out[0],
                           token_out=out[1], workspace=ws)
        dvs.sample_filtered(zvt[:, 0], u0, d["T"], d["k"],
                            d["p"], d["m"], token_out=out[2], prob_out=pr)

    u0 = ut[:, 0].clone()
    step()
    torch.cuda.synchronize()
    g = dvs.capture(step)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(4):
        ut.copy_(torch.rand(ut.shape, device="cuda", generator=gen))
        u0.copy_(ut[:, 0])
        zvt.copy_(zvt.flip(0))
        g.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in out] + [pr.clone()]
        torch.randn(1 << 20, device="cuda").sum().item()
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, out + [pr]):
            assert torch.equal(a, b)


def test_other_stream():
    rows, V = 8, 20011
    rng = np.random.default_rng(12)
    zt, z64 = _rounded(_logits("normal", rows, V, rng), "f32")
    par = _params(rows)
    d = _dev(par)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got_t, got_p = _call(zt, d)
    s.synchronize()
    _check(z64, par, got_t.cpu().numpy(), got_p.cpu().numpy())


def test_binding_refusals():
    z = torch.zeros(4, 8, device="cuda")
    u = torch.zeros(4, device="cuda")
    f = lambda n: torch.ones(n, device="cuda")   # noqa: E731
    for bad in (lambda: dvs.sample_filtered(z.half(), u),
                lambda: dvs.sample_filtered(z, u[:3]),
                lambda: dvs.sample_filtered(z.t(), torch.zeros(8, device="cuda")),
                lambda: dvs.sample_filtered(z, u, temperature=f(3)),
                lambda: dvs.sample_filtered(z, u, temperature=f(4), top_p=f(2)),
                lambda: dvs.sample_filtered(z, u, top_k=f(4)),
                lambda: dvs.sample_filtered(z[:1].expand(4, 8), u),
                lambda: dvs.sample_filtered(z.view(2, 2, 8)[:, :, :4], u.view(2, 2)),
                lambda: dvs.accept_sampled(z.view(1, 4, 8), z[:2].view(1, 2, 8),
                                           torch.zeros(1, 2, dtype=torch.int32, device="cuda"), u),
                lambda: dvs.accept_sampled(z[:3].view(1, 3, 8), z[:2].view(1, 2, 8),
                                           torch.zeros(1, 1, dtype=torch.int32, device="cuda"),
                                           torch.zeros(1, 3, device="cuda"))):
        with pytest.raises(dvs.DvsError):
            bad()
