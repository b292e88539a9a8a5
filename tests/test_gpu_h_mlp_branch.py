"""The example that runs the block operators and the int8 history together, against the same blocks in 64 bits.

Bounds of a branch's relative error (2-norm), from the formats: e4m3 rows are off by at most 2^-4 of themselves and evenly so,
2^-4 / sqrt(3) = 3.6e-2 (the weights are taken as they are), and products of independent errors keep that size; GELU's
slope against its value may raise it by half; bf16 adds 2e-3. A prediction with the weights w = (3, -10, 15) / 8 of half a
spacing past three nodes raises an error of its entries by |w| = 2.3 against entries that agree to a few per cent, and the
history's step, 1/254 of a block's largest value (2.7 deviations of 64), adds 6.1e-3 |w| of it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("depth,batch,tokens,hidden", [(1, 2, 77, 768), (4, 2, 256, 1152), (3, 3, 50, 136)])
def test_example(depth, batch, tokens, hidden):
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import mlp_branch
    m, off = mlp_branch.run(depth, batch, tokens, hidden, dtype=torch.float64)
    m.close()
    branch = 1.5 * 3.6e-2 + 2e-3
    for t, rel, change in off[:-1]:
        assert change < branch, (t, rel, change)
    assert off[-1][2] < 2.3 * (branch + 6.1e-3), off[-1]


def test_depth_is_checked():
    from paper_2608_23429_gb300 import mlp_branch
    with pytest.raises(ValueError):
        mlp_branch.MlpBranches(5, 1, 1, 64, [2.0, 1.0])
