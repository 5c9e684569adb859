"""GPU: attn_tree over batches of hundreds of sequences, whose lengths every wave of a workgroup
counts, with the tiles through LDS and without; rows whose scores are all -inf."""
import numpy as np
import pytest

from oracle import tree as ot
from paper_2609_26638_amd import dvs
from tests.gpu_util import to_f64
from tests.test_gpu_tree_append import dev, i32
from tests.test_gpu_tree_attn import run
from tests.tree_util import cache, random_parents, rounded

pytestmark = pytest.mark.gpu

# S, R, Hq, Hkv, D: more than 32 rows of a KV head (tiles through LDS in short tables and in wide
# ones) or fewer, and lengths in every group of 64 sequences
CASES = [(257, 20, 4, 2, 64), (513, 17, 4, 2, 64), (600, 35, 2, 2, 64), (1024, 33, 2, 2, 64),
         (320, 20, 8, 4, 128), (450, 18, 6, 3, 96), (1030, 40, 2, 2, 64), (700, 5, 4, 2, 64),
         (1024, 2, 4, 1, 96)]


@pytest.mark.parametrize("columns", [0, 300])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"S{c[0]}R{c[1]}H{c[2]}-{c[3]}D{c[4]}")
def test_hundreds_of_sequences(case, columns):
    S, R, *rest = case
    rng = np.random.default_rng(S + R)
    lens = [int(x) for x in rng.integers(1, 150, S)]
    lens[S // 2] = lens[S - 1] = 0
    lens[S // 3] = 260
    parent = random_parents(rng, S, R)
    vis, _, _ = ot.masks(parent)
    run((lens, R, *rest), "bf16", vis, dvs.tree_masks(i32(parent))[0], columns=columns)


@pytest.mark.parametrize("case", [(257, 20, 4, 2, 64), (1024, 3, 4, 2, 64)],
                         ids=lambda c: f"S{c[0]}R{c[1]}H{c[2]}-{c[3]}D{c[4]}")
def test_hundreds_of_sequences_fp32(case):
    S, R, *rest = case
    rng = np.random.default_rng(S)
    lens = [int(x) for x in rng.integers(0, 150, S)]
    vis, _, _ = ot.masks(random_parents(rng, S, R))
    run((lens, R, *rest), "f32", vis, i32(ot.words(vis)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("columns", [0, 1100])
@pytest.mark.parametrize("R,Hq,Hkv,D", [(3, 4, 2, 64), (40, 8, 2, 128), (20, 4, 1, 96)])
def test_rows_with_scores_of_minus_infinity_only(R, Hq, Hkv, D, columns, dtype):
    """3e38 * -4 leaves 32 bits: such a row gives 0, the rows beside it what they give without it."""
    lens = [300, 45]
    st, k, v = cache(R, lens, R, Hkv, D, dtype)
    k[..., 0] = -4
    rng = np.random.default_rng(R)
    q = rounded(rng.standard_normal((2, R, Hq, D)), dtype)
    parent = random_parents(rng, 2, R, padding=False)
    table = np.pad(st.page_table, ((0, 0), (0, max(0, columns - st.page_table.shape[1]))))
    args = (dev(k, dtype), dev(v, dtype), i32(table), i32(st.kv_len), dvs.tree_masks(i32(parent))[0], D ** -0.5)
    want = to_f64(dvs.attn_tree(dev(q, dtype), *args))
    row = R // 2
    q[:, row] = 0
    q[:, row, :, 0] = rounded(3e38, dtype)
    got = to_f64(dvs.attn_tree(dev(q, dtype), *args))
    assert np.all(got[:, row] == 0)
    others = np.arange(R) != row
    np.testing.assert_array_equal(got[:, others], want[:, others])
