"""The example that runs the codec and the attention entry points together."""
import pytest

from paper_2507_17511_amd import ring_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("peers,tokens,q_heads,kv_heads,dim", [(4, 512, 8, 8, 128), (3, 300, 6, 2, 64), (2, 130, 4, 1, 256)])
def test_ring_attention_and_decoding(peers, tokens, q_heads, kv_heads, dim):
    same, exact, decoded = ring_attention.run(peers, tokens, q_heads, kv_heads, dim, steps=3, decode=3, page_size=16, say=lambda *_: None)
    # bf16 weights, parts and outputs are rounded, each by about 0.0016 of its size on the whole (2^-7 / sqrt(12) of the leading power of two):
    # three of them at random make 0.0028
    assert same < 2.0 ** -8 and decoded < 2.0 ** -8
    # the codec's error on top: 2-bit residuals of a drift of 0.03, which error feedback keeps from growing
    assert exact < 0.1
