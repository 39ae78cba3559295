"""The attention profile's request selection (no GPU needed)."""
import os

import numpy as np
import pytest

pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2512_14098_amd", "libcf.so")),
                                reason="libcf.so not built")


def test_component_tokens_of_the_omni_graph():
    """Input tokens of each component: its selected attributes summed, audio at 80 ms a token,
    over the requests whose type runs it."""
    from paper_2512_14098_amd.attn_profile import component_tokens
    from paper_2512_14098_amd.inputs import load_config
    model = load_config("c2")["model"]
    z = np.zeros(4, np.int64)
    trace = dict(type=np.array([0, 1, 2, 3]), prompt=np.array([10, 20, 30, 40]), out=np.array([1, 2, 3, 0]),
                 patches=np.array([0, 300, 0, 500]), aud_in_ms=np.array([0, 0, 81, 160]), aud_out_ms=z + 240)
    x, out = component_tokens(model, trace, "L_th")
    assert x.tolist() == [10, 320, 32, 542] and out.tolist() == [1, 2, 3, 1]
    x, out = component_tokens(model, trace, "L_ta")
    assert x.tolist() == [30, 40] and out.tolist() == [3, 3]
    assert component_tokens(model, trace, "E_img")[0].tolist() == [300, 500]
