"""The example runs the operators with the framework's exchange, as a user would."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ranks,tokens,hidden,inter,k", [(8, 64, 256, 128, 2), (6, 5, 144, 80, 3), (64, 32, 512, 256, 2)])
def test_dispatch_experts_and_return(ranks, tokens, hidden, inter, k):
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import moe_layer
    same, near = moe_layer.main(["--ranks", str(ranks), "--tokens", str(tokens), "--hidden", str(hidden), "--inter", str(inter), "--k", str(k)])
    assert same            # through the exchange and back, bit for bit
    assert near < 0.1      # x and h in 8 bits (2^-4 a value, averaged over the row) against 16
