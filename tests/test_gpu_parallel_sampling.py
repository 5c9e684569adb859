"""GPU: filtered rounds, and several sampled continuations of one prefix from
prefill to compaction.

* literal_round_filtered against the oracle's sampled round over filtered
  distributions, on the same uniforms (decision margins recorded, as for
  literal_round_sampled); with T = 0 it commits the greedy AR stream.
* A prefilled slot is forked, every slot decodes on its own, slots are
  released and refilled, the pool is compacted: each slot's stream equals the
  one of a state in which its sequence was prefilled and decoded alone."""
import numpy as np
import pytest
import torch

from oracle import filter as of
from oracle.model import OracleModel
from paper_2609_26638_amd import dvs, synth
from tests.test_gpu_diffusion import _model_and_state
from tests.test_gpu_model_step import _dev_pools, _states_equal
from tests.test_gpu_sampling import _cdf_margin

pytestmark = pytest.mark.gpu


def _params(S):
    return dict(temperature=np.linspace(0.6, 1.2, S).astype(np.float32),
                top_k=(np.arange(S, dtype=np.int32) % 3) * 20,
                top_p=np.linspace(0.99, 0.8, S).astype(np.float32),
                min_p=np.where(np.arange(S) % 2, 0.02, 0.0).astype(np.float32))


def _dev(par):
    return {n: torch.from_numpy(a).cuda() for n, a in par.items()}


def _kept(par, s, z):
    return of.kept_weights(z, float(par["temperature"][s]), int(par["top_k"][s]),
                           float(par["top_p"][s]), float(par["min_p"][s]))


def _cut_margin(par, s, z):
    """Largest error E of a row's logits that cannot change its kept set.  Top-k:
    two logits move towards each other by 2 E at most.  Top-p: the share c of a
    prefix moves by sum w_i e_i (1 - c) / T - ... <= 2 E c (1 - c) / T.  Min-p:
    a weight moves by 2 E / T of itself."""
    T, k, p, m = (float(par[n][s]) for n in ("temperature", "top_k", "top_p", "min_p"))
    o = np.sort(z)[::-1]
    w = np.exp((o - o[0]) / T)
    mg = np.inf
    n = len(w)
    if 0 < k < n:
        n = int(k)
        mg = min(mg, (o[n - 1] - o[n]) / 2)
    if p < 1:
        c = np.cumsum(w[:n])
        mg = min(mg, np.abs(c / c[-1] - p).min() * T / (2 * p * (1 - p)))
    if m > 0:
        mg = min(mg, np.abs(w / m - 1).min() * T / 2)
    return mg


def test_filtered_round_matches_oracle():
    B = 6
    w, host, kps, vps = _model_and_state("f32", B, seed=28)
    host.draft = np.zeros((host.kv_len.shape[0], B), np.int32)
    S = host.kv_len.shape[0]
    om = OracleModel(w, kps, vps)
    dm = dvs.DeviceModel(w, _dev_pools(kps, "f32"), _dev_pools(vps, "f32"), "f32")
    st, ref, par = dvs.DeviceState(host), host.copy(), _params(S)
    d, acc = _dev(par), torch.empty(S, dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(3)
    for rnd in range(2):
        u = rng.random((S, 2 * B + 2)).astype(np.float32)
        u64 = u.astype(np.float64)
        lg_d, lg_v, A, final, err = om.sampled_round(
            ref, B, 1.0, u64, dist=lambda s, z: of.probs(_kept(par, s, z)))
        assert err == 0
        mg = np.inf
        for s in range(S):
            pv = np.array([of.probs(_kept(par, s, lg_v[s, r])) for r in range(B + 1)])
            qd = np.array([of.probs(_kept(par, s, lg_d[s, r])) for r in range(B + 1)])
            for r in range(B + 1):
                mg = min(mg, _cdf_margin(qd[r], u64[s, r]), _cut_margin(par, s, lg_d[s, r]))
            for r in range(int(A[s]) + 1):
                mg = min(mg, _cut_margin(par, s, lg_v[s, r]))
            t = [of.draw(qd[r], u64[s, r]) for r in range(B + 1)]
            for j in range(1, min(int(A[s]) + 1, B) + 1):
                a, b = pv[j - 1][t[j]], qd[j][t[j]]
                mg = min(mg, abs(u64[s, B + j] * b - a) / max(a, b))
            a = int(A[s])
            wt = pv[a] if a == B else np.maximum(pv[a] - qd[a + 1], 0)
            mg = min(mg, _cdf_margin(wt, u64[s, 2 * B + 1]))
            assert of.accept(pv, qd[1:], np.array(t[1:]), u64[s, B + 1:]) == (a, int(final[s]))
        print(f"[round {rnd}] A={list(A)} smallest decision margin {mg:.3e}")
        # fp32 logits are within ~2e-6 of the row's largest |logit| (~1 here)
        assert mg > 1e-5
        dvs.literal_round_filtered(dm, st, B, torch.from_numpy(u).cuda(), **d, accept_out=acc)
        torch.cuda.synchronize()
        assert int(st.err.item()) == 0
        np.testing.assert_array_equal(acc.cpu().numpy(), A)
        _states_equal(st, ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("greedy", ["temperature", "top_k", "min_p"])
def test_greedy_filters_commit_the_ar_stream(dtype, greedy):
    B, N, CH = 8, 24, 64
    w, host, kps, vps = _model_and_state(dtype, B)
    host.draft = np.zeros((host.kv_len.shape[0], B), np.int32)
    S = host.kv_len.shape[0]
    ar_m = dvs.DeviceModel(w, _dev_pools(kps, dtype), _dev_pools(vps, dtype), dtype)
    ar_st = dvs.DeviceState(host)
    for _ in range(N):
        dvs.draft_verify_step(ar_m, ar_st, 1, 0, chunk_keys=CH)
    sm = dvs.DeviceModel(w, _dev_pools(kps, dtype), _dev_pools(vps, dtype), dtype)
    ss = dvs.DeviceState(host)
    par = {"temperature": dict(temperature=torch.zeros(S, device="cuda")),
           "top_k": dict(top_k=torch.ones(S, dtype=torch.int32, device="cuda")),
           "min_p": dict(min_p=torch.full((S,), 1.5, device="cuda"))}[greedy]
    gen = torch.Generator(device="cuda").manual_seed(5)
    rounds = 0
    while int(ss.out_count.min().item()) < N:
        u = torch.rand((S, 2 * B + 2), device="cuda", generator=gen)
        dvs.literal_round_filtered(sm, ss, B, u, **par, chunk_keys=CH)
        rounds += 1
        assert rounds <= N
    torch.cuda.synchronize()
    assert int(ar_st.err.item()) == 0 and int(ss.err.item()) == 0
    ar, sr = ar_st.to_host(host), ss.to_host(host)
    for s in range(S):
        n = min(int(sr.out_count[s]), int(ar.out_count[s]))
        assert n >= N
        np.testing.assert_array_equal(sr.out_tokens[s, :n], ar.out_tokens[s, :n])


def test_parallel_continuations():
    B, CH, S, P = 4, 64, 4, 37
    W = B + 2
    w = synth.make_model_weights(11, 512, 256, 4, 2, 64, 2, 512, std=0.08)
    rng = np.random.default_rng(2)
    prompts = [rng.integers(0, 512, (1, P)).astype(np.int32) for _ in range(2)]
    par = _params(S)
    us = rng.random((40, S, 2 * B + 2)).astype(np.float32)

    def fresh(n):
        st = synth.make_paged_state(rng, np.full(n, P), W, 12, True, extra_pages=80, n_causal=B + 1,
                                    max_new=64)
        st.kv_len[:] = 0
        pools = [[torch.zeros((st.pool_pages, 2) + p, dtype=torch.bfloat16, device="cuda")
                  for _ in range(2)] for p in ((16, 64), (64, 16))]
        m = dvs.DeviceModel(w, pools[0], pools[1], "bf16")
        return m, dvs.DeviceState(st), dvs.KVPools(*pools), st

    def rounds(m, st, first, count, rows):
        for i in range(first, first + count):
            dvs.literal_round_filtered(m, st, B, torch.from_numpy(us[i][rows]).cuda(),
                                       **{n: torch.from_numpy(a[rows]).cuda()
                                          for n, a in par.items()}, chunk_keys=CH)

    def alone(prompt, slot, first, count):
        m, st, _, host = fresh(1)
        dvs.prefill(m, st, P, B, torch.from_numpy(prompt).cuda(), chunk_keys=CH)
        rounds(m, st, first, count, [slot])
        torch.cuda.synchronize()
        assert int(st.err.item()) == 0
        return st.to_host(host)

    def check(got, s, want):
        n = int(want.out_count[0])
        assert int(got.out_count[s]) == n and int(got.kv_len[s]) == int(want.kv_len[0])
        np.testing.assert_array_equal(got.out_tokens[s, :n], want.out_tokens[0, :n])

    ids = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")   # noqa: E731
    m, st, pools, host = fresh(S)
    dvs.kv_release(st, ids(0, 1, 2, 3), W)
    dvs.kv_release(st, ids(0), P + W)
    dvs.prefill(m, st.slots(0, 1), P, B, torch.from_numpy(prompts[0]).cuda(), chunk_keys=CH)
    dvs.kv_fork(st, pools, ids(0, 0, 0), ids(1, 2, 3), W)
    assert int(st.page_refs.sum()) == 3 * (P // 16)
    rounds(m, st, 0, 5, [0, 1, 2, 3])
    torch.cuda.synchronize()
    assert int(st.err.item()) == 0
    got = st.to_host(host)
    for s in range(S):
        check(got, s, alone(prompts[0], s, 0, 5))
    # the source and another go; slot 0 takes a second document; compaction
    dvs.kv_release(st, ids(0, 2), P + W)
    moved = dvs.kv_compact(st, pools)
    assert int(st.err.item()) == 0 and int(moved.item()) > 0
    dvs.prefill(m, st.slots(0, 1), P, B, torch.from_numpy(prompts[1]).cuda(), chunk_keys=CH)
    rounds(m, st, 5, 4, [0, 1, 2, 3])
    dvs.kv_compact(st, pools)
    rounds(m, st, 9, 2, [0, 1, 2, 3])
    torch.cuda.synchronize()
    assert int(st.err.item()) == 0
    got = st.to_host(host)
    for s in (1, 3):
        check(got, s, alone(prompts[0], s, 0, 11))
    check(got, 0, alone(prompts[1], 0, 5, 6))
    assert int(got.out_count[2]) == 0 and int(got.kv_len[2]) == 0 and int(got.finished[2]) == 1
    used = st.pool_pages - got.free_top
    assert got.page_table.max() < st.pool_pages and used > 0
