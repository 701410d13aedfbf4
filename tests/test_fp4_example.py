"""The example with 4-bit weights, around the framework's exchange."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ranks,tokens,hidden,inter,k", [(8, 64, 256, 128, 2), (6, 5, 160, 96, 3), (64, 32, 512, 256, 2)])
def test_dispatch_experts_and_return(ranks, tokens, hidden, inter, k):
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import moe_layer
    same, near = moe_layer.main(["--ranks", str(ranks), "--tokens", str(tokens), "--hidden", str(hidden), "--inter", str(inter), "--k", str(k), "--bits", "4"])
    assert same            # through the exchange and back, bit for bit
    assert near < 0.01     # the same calls on fewer rows: only the router's product may round otherwise
