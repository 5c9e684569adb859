"""GPU: acceptance over rows with ties, equal and masked logits, and drafts outside
the kept tokens, against the oracle; filtered rounds without filters against
literal_round_sampled, which computes its softmax in fp32.

Decisions: u is a multiple of 2^-24 drawn at random, so that u q = p, or u W on
the border of a token, has to be met to within the 64-bit sums' roundings; for
the fp32 softmax, to 1e-6 of the row's weight, once in some 10^5 draws."""
import numpy as np
import pytest
import torch

from oracle import filter as of
from paper_2609_26638_amd import dvs
from tests.test_gpu_diffusion import _model_and_state
from tests.test_gpu_filter import _logits, _params, _rounded
from tests.test_gpu_model_step import _dev_pools, _states_equal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["levels", "equal", "masked", "spread", "flat"])
@pytest.mark.parametrize("S,B,V", [(9, 3, 5), (11, 5, 301), (7, 2, 4099), (60, 4, 1021), (4, 2, 20011)])
def test_ties_and_masks(S, B, V, kind, dtype):
    rng = np.random.default_rng([S, B, V, len(kind)])
    zv = _logits(kind, S * (B + 1), V, rng).reshape(S, B + 1, V)
    zd = _logits(kind, S * B, V, rng).reshape(S, B, V)
    same = rng.random((S, B)) < 0.6                # most drafts come from the verifier's row
    zd[same] = zv[:, :B][same]
    zvt, zv64 = _rounded(zv, dtype)
    zdt, zd64 = _rounded(zd, dtype)
    par = _params(S)
    par["T"] = np.where(np.arange(S) % 5 == 4, 0.0, rng.uniform(0.5, 1.5, S)).astype(np.float32)
    par["k"] = np.array([0, 3, 0, 40, 700][:S] * S, np.int32)[:S]
    dist = lambda z, s: of.probs(of.kept_weights(z, float(par["T"][s]), int(par["k"][s]),   # noqa: E731
                                                 float(par["p"][s]), float(par["m"][s])))
    u = rng.random((S, B + 1)).astype(np.float32)
    draft, want = np.zeros((S, B), np.int32), []
    for s in range(S):
        pv = np.array([dist(z, s) for z in zv64[s]])
        qd = np.array([dist(z, s) for z in zd64[s]])
        draft[s] = [of.draw(q, rng.random()) for q in qd]
        if s % 4 == 3:
            draft[s, B - 1] = rng.integers(-2, V + 2)
        want.append(of.accept(pv, qd, draft[s], u[s].astype(np.float64), zv64[s]))
    d = {n: torch.from_numpy(par[n]).cuda() for n in "Tkpm"}
    A, tok = dvs.accept_sampled(zvt, zdt, torch.from_numpy(draft).cuda(),
                                torch.from_numpy(u).cuda(), d["T"], d["k"], d["p"], d["m"])
    assert list(zip(A.tolist(), tok.tolist())) == want


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [0.7, 1.0])
def test_rounds_without_filters(T, dtype):
    B, CH, N = 6, 64, 8
    w, host, kps, vps = _model_and_state(dtype, B, seed=31)
    host.draft = np.zeros((host.kv_len.shape[0], B), np.int32)
    S = host.kv_len.shape[0]
    make = lambda: (dvs.DeviceModel(w, _dev_pools(kps, dtype), _dev_pools(vps, dtype), dtype),   # noqa: E731
                    dvs.DeviceState(host), torch.empty(S, dtype=torch.int32, device="cuda"))
    (fm, fs, fa), (sm, ss, sa) = make(), make()
    temp = torch.full((S,), T, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(11)
    for _ in range(N):
        u = torch.rand((S, 2 * B + 2), device="cuda", generator=gen)
        dvs.literal_round_filtered(fm, fs, B, u, temperature=temp, chunk_keys=CH, accept_out=fa)
        dvs.literal_round_sampled(sm, ss, B, float(np.float32(T)), u, chunk_keys=CH, accept_out=sa)
        torch.cuda.synchronize()
        assert int(fs.err.item()) == 0 and int(ss.err.item()) == 0
        assert fa.tolist() == sa.tolist()
        _states_equal(fs, ss.to_host(host))


@pytest.mark.parametrize("filters", ["top_k", "top_p", "all"])
def test_bf16_rounds_follow_their_logits(filters):
    """A bf16 model's round, replayed from its verify logits: accepted drafts are
    kept tokens of their rows, and the final token of sequences that accept all
    is the oracle's draw."""
    B, CH, N = 4, 64, 6
    w, host, kps, vps = _model_and_state("bf16", B, seed=33)
    host.draft = np.zeros((host.kv_len.shape[0], B), np.int32)
    S = host.kv_len.shape[0]
    m = dvs.DeviceModel(w, _dev_pools(kps, "bf16"), _dev_pools(vps, "bf16"), "bf16")
    st = dvs.DeviceState(host)
    par = {}
    if filters != "top_p":
        par["top_k"] = np.full(S, 40, np.int32)
    if filters != "top_k":
        par["top_p"] = np.full(S, 0.95, np.float32)
    if filters == "all":
        par["min_p"] = np.full(S, 0.01, np.float32)
    d = {n: torch.from_numpy(a).cuda() for n, a in par.items()}
    logits = torch.empty((S, B + 1, w.V), device="cuda")
    acc = torch.empty(S, dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(2)
    before = np.zeros(S, np.int64)
    for _ in range(N):
        u = torch.rand((S, 2 * B + 2), device="cuda", generator=gen)
        dvs.literal_round_filtered(m, st, B, u, **d, chunk_keys=CH, logits_out=logits, accept_out=acc)
        torch.cuda.synchronize()
        assert int(st.err.item()) == 0
        got, z, A = st.to_host(host), logits.double().cpu().numpy(), acc.tolist()
        for s in range(S):
            kept = [of.kept_weights(z[s, r], 1.0, int(par.get("top_k", [0] * S)[s]),
                                    float(par.get("top_p", [1.0] * S)[s]),
                                    float(par.get("min_p", [0.0] * S)[s])) for r in range(B + 1)]
            new = got.out_tokens[s, before[s]:got.out_count[s]].tolist()   # a0, d_1..d_A, final
            before[s] = got.out_count[s]
            if got.finished[s]:
                continue
            assert len(new) == A[s] + 2 and new[1:-1] == got.draft[s, :A[s]].tolist()
            assert all(kept[r][t] > 0 for r, t in enumerate(new[1:]))
            if A[s] == B:
                assert new[-1] == of.draw(kept[B], float(u[s, 2 * B + 1]))
