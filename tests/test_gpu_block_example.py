"""The block's calls and the 8-bit layer together, as the example runs them: a stack learns, and serves what it has learnt."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_the_stack_learns_and_is_served():
    from examples import decoder_block

    torch.manual_seed(0)
    losses, apart = decoder_block.main(steps=30)
    # a residual stream of unit rows against unit targets: 2 and what the blocks add; each token id's row can be learnt
    assert losses[-1] < 0.8 * losses[0]
    # 8 bits in four operands of each of two blocks: 0.7 to 2.3 % of the branch each
    assert max(apart) < 0.05
