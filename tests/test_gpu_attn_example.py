"""The example that runs the attention operators between two delta linears, as a user would."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.gpu
@pytest.mark.parametrize("q_heads,kv_heads,head_dim", [(8, 2, 128), (4, 4, 64)])
def test_decoding_over_the_cache_agrees_with_longer_prompts(q_heads, kv_heads, head_dim):
    """A code is off by at most half a step of amax / 127: about 0.9 % of a normal value's deviation (amax of a page's thousands
    of values is near 4 deviations: 4 / 127 / sqrt(12)).  Weights of averages over independent tokens scale signal and error
    alike, scores move by the same fraction of their deviation; 3 % leaves room for both and for codes rounded again."""
    import decoder_block
    off = decoder_block.run(q_heads, kv_heads, head_dim, lens=(90, 1, 200), steps=5)
    assert 0 < off < 0.03, off
