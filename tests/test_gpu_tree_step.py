"""GPU: the tree step's calls together, as a decoder uses them: masks, append, attention, top-1,
commit, over several steps; on streams of their own, captured and replayed."""
import math

import numpy as np
import pytest
import torch

from oracle import tree as ot
from paper_2609_26638_amd import dvs
from tests.gpu_util import to_f64
from tests.test_gpu_tree_append import dev, i32
from tests.test_gpu_tree_attn import check
from tests.tree_util import cache, random_parents, rounded

pytestmark = pytest.mark.gpu

S, R, HQ, HKV, D, V, LAYERS = 3, 18, 4, 2, 64, 24, 2


class Decoder:
    """A toy decoder: each token has fixed queries, keys and values a layer, and the logits are
    products of the last layer's output with fixed vectors."""

    def __init__(self, dtype, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        tt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.table = torch.randn((LAYERS, V, (HQ + 2 * HKV) * D), device="cuda", generator=g).to(tt)
        self.head = torch.randn((HQ * D, V), device="cuda", generator=g)
        st, k, v = cache(seed, [21, 0, 40], R, HKV, D, dtype)
        st.out_tokens = np.full((S, 200), -1, np.int32)
        # room for a few steps
        self.state = dvs.DeviceState(st)
        self.k = [dev(k, dtype) for _ in range(LAYERS)]
        self.v = [dev(v, dtype) for _ in range(LAYERS)]
        self.pools = dvs.KVPools(self.k, self.v)
        self.attn_ws = dvs.Workspace(dvs.tree_workspace_bytes(S, R, HQ, HKV, D, st.max_pages, tt))
        self.ws = dvs.Workspace(dvs.accept_tree_workspace_bytes(S, R))

    def forward(self, tokens, parent):
        """The verifier's logits for every row, by the framework's calls."""
        s = self.state
        mask, depth = dvs.tree_masks(parent, err=s.err)
        for l in range(LAYERS):
            x = self.table[l][tokens.long()]
            q, k, v = (t.unflatten(-1, (-1, D)) for t in x.split([HQ * D, HKV * D, HKV * D], -1))
            q = dvs.kv_append_rope(q, k, v, self.k[l], self.v[l], s.page_table, s.kv_len,
                                   depth=depth, err=s.err)
            o = dvs.attn_tree(q, self.k[l], self.v[l], s.page_table, s.kv_len, mask,
                              1 / math.sqrt(D), err=s.err, workspace=self.attn_ws)
        return o.flatten(2).float() @ self.head

    def step(self, tokens, parent, out=None):
        z = self.forward(tokens, parent)
        am = dvs.argmax_accept(z, R, self.none(), accept=False)[0]
        return dvs.accept_commit_tree(self.state, self.pools, parent, tokens, am,
                                      workspace=self.ws), am

    def none(self):
        if not hasattr(self, "_none"):
            self._none = torch.zeros((S, R), dtype=torch.int32, device="cuda")
        return self._none


def trees(rng, bound):
    """Random trees whose row 0 is each sequence's boundary token."""
    parent = random_parents(rng, S, R)
    tokens = rng.integers(0, V, (S, R))
    tokens[:, 0] = bound
    return tokens, parent


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_decode_what_single_tokens_decode(dtype):
    """The committed tokens are those of greedy decoding a token at a time through the same
    calls (R = 1), as far as its top-1 is clear of the rounding."""
    rng = np.random.default_rng(1)
    a = Decoder(dtype)
    boundary = torch.tensor([3, 1, 2], dtype=torch.int32, device="cuda")
    a.state.boundary.copy_(boundary)
    for _ in range(4):
        tokens, parent = trees(rng, a.state.boundary.cpu().numpy())
        a.step(i32(tokens), i32(parent))
    assert int(a.state.err) == 0
    count = a.state.out_count.cpu().numpy()
    out = a.state.out_tokens.cpu().numpy()
    assert count.sum() >= 4 * S                       # a token a step at least
    # greedy decoding: one row, no mask, no depth
    b = Decoder(dtype)
    cur = boundary.clone()
    live = np.ones(S, bool)
    for i in range(int(count.max())):
        s = b.state
        for l in range(LAYERS):
            x = b.table[l][cur.long().view(S, 1)]
            q, k, v = (t.unflatten(-1, (-1, D)) for t in x.split([HQ * D, HKV * D, HKV * D], -1))
            q = dvs.kv_append_rope(q, k, v, b.k[l], b.v[l], s.page_table, s.kv_len)
            o = dvs.attn_tree(q, b.k[l], b.v[l], s.page_table, s.kv_len, None, 1 / math.sqrt(D))
        z = (o.flatten(2).float() @ b.head)[:, 0]
        top = z.topk(2, -1)
        s.kv_len += 1
        # 2^-6 of the largest logit: several times what roundings of 2^-8 leave
        live &= ((top.values[:, 0] - top.values[:, 1]) > 2.0 ** -6 * z.abs().amax(-1)).cpu().numpy()
        nxt = top.indices[:, 0].to(torch.int32)
        for q in range(S):
            if live[q] and i < count[q]:
                assert int(nxt[q]) == out[q, i], (q, i)
        # go on from what was committed
        cur = torch.where(i32(i < count) > 0, i32(out[:, i]), nxt)
        live |= i < count


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_cache_after_a_step_is_that_of_the_path(dtype):
    """After commits by trees, the cache holds what appending the committed tokens in a row
    gives, bit for bit, and attention over it is the oracle's."""
    rng = np.random.default_rng(2)
    a = Decoder(dtype, seed=4)
    before = [int(x) for x in a.state.kv_len]
    stream = [[] for _ in range(S)]                   # the tokens whose slots are committed
    for _ in range(3):
        tokens, parent = trees(rng, a.state.boundary.cpu().numpy())
        (took, path), _ = a.step(i32(tokens), i32(parent))
        for s in range(S):
            stream[s] += [int(tokens[s, r]) for r in path[s, :int(took[s]) + 1].cpu()]
    kv_len, pt = a.state.kv_len.cpu().numpy(), a.state.page_table.cpu().numpy()
    b = Decoder(dtype, seed=4)                        # the same initial cache
    for s in range(S):
        n = len(stream[s])
        assert kv_len[s] == before[s] + n
        for l in range(LAYERS):
            x = b.table[l][torch.tensor(stream[s], device="cuda")].view(1, n, -1)
            q, k, v = (t.unflatten(-1, (-1, D)) for t in x.split([HQ * D, HKV * D, HKV * D], -1))
            ids = i32(pt[s:s + 1])
            dvs.kv_append_rope(q, k, v, b.k[l], b.v[l], ids, i32([before[s]]))
            for t in range(before[s], before[s] + n):
                pg, sl = pt[s, t // 16], t % 16
                assert torch.equal(a.k[l][pg, :, sl], b.k[l][pg, :, sl])
                assert torch.equal(a.v[l][pg, :, :, sl], b.v[l][pg, :, :, sl])
    q = rounded(rng.standard_normal((S, 1, HQ, D)), dtype)
    a.state.kv_len.sub_(1)                            # the last committed token as the window
    got = to_f64(dvs.attn_tree(dev(q, dtype), a.k[0], a.v[0], a.state.page_table, a.state.kv_len,
                               None, 0.125))
    want, size = ot.attention(q.astype(float), to_f64(a.k[0]), to_f64(a.v[0]), pt, kv_len - 1,
                              np.ones((S, 1, 1), bool), 0.125)
    check(got, want, size, dtype)


def fields(d):
    return [getattr(d.state, f).clone() for f in dvs.DeviceState.FIELDS] + \
        [d.state.free_top.clone()] + [t.clone() for t in d.k + d.v]


def test_captured_steps_replay_as_eager_ones():
    """Two graphs that share the workspaces, replayed in turn with eager work between, against
    the same steps run eagerly."""
    rng = np.random.default_rng(5)
    eager, graph = Decoder("bf16", 7), Decoder("bf16", 7)
    sets = [(i32(t), i32(p)) for t, p in (trees(rng, 0) for _ in range(2))]
    for d in (eager, graph):
        d.step(*sets[0])                              # warm
    torch.cuda.synchronize()
    outs = []
    graphs = [dvs.capture(lambda s=s: outs.append(graph.step(*s))) for s in sets]
    for i in range(6):
        graphs[i % 2].replay()
        want = eager.step(*sets[i % 2])
        junk = torch.randn(1 << 18, device="cuda").sum()
        torch.cuda.synchronize()
        assert float(junk) == float(junk)
        (acc, path), am = outs[i % 2]
        (wacc, wpath), wam = want
        assert torch.equal(acc, wacc) and torch.equal(path, wpath) and torch.equal(am, wam)
        for x, y in zip(fields(graph), fields(eager)):
            assert torch.equal(x, y)
    assert int(graph.state.err) == 0


def test_calls_on_a_stream_of_their_own():
    """Outputs and scratch that a call makes belong to the stream it is given, while other work
    keeps the current stream busy."""
    rng = np.random.default_rng(6)
    tokens, parent = (i32(x) for x in trees(rng, 0))
    ref = Decoder("bf16", 3)
    want = ref.forward(tokens, parent)
    d = Decoder("bf16", 3)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = torch.randn((2048, 2048), device="cuda")
    for _ in range(8):
        busy = busy @ busy * 1e-3                     # on the current stream
    s = d.state
    with torch.cuda.stream(side):
        xs = [d.table[l][tokens.long()] for l in range(LAYERS)]
    mask, depth = dvs.tree_masks(parent, stream=side)
    for l in range(LAYERS):
        q, k, v = (t.unflatten(-1, (-1, D)) for t in xs[l].split([HQ * D, HKV * D, HKV * D], -1))
        q = dvs.kv_append_rope(q, k, v, d.k[l], d.v[l], s.page_table, s.kv_len, depth=depth,
                               stream=side)
        o = dvs.attn_tree(q, d.k[l], d.v[l], s.page_table, s.kv_len, mask, 1 / math.sqrt(D),
                          stream=side)
    side.synchronize()
    got = o.flatten(2).float() @ d.head
    assert torch.equal(got, want)
    (acc, path), am = ref.step(tokens, parent)
    acc2, path2 = dvs.accept_commit_tree(s, d.pools, parent, tokens, am, stream=side)
    side.synchronize()
    assert torch.equal(acc, acc2) and torch.equal(path, path2)
    for x, y in zip(fields(d), fields(ref)):
        assert torch.equal(x, y)
