"""The sequences that an encoder's profile attends over: every image of a request on its own."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("config,component,seed", [("c1", "E", 0), ("c1", "E", 2 ** 64 - 3), ("c2", "E_img", 7)])
def test_each_image_is_a_sequence(monkeypatch, config, component, seed):
    """As many sequences as images, each of a length that an image may have, a request's images
    adding up to its patches in the trace."""
    from paper_2512_14098_amd import attn_profile as A
    from paper_2512_14098_amd import cf
    from paper_2512_14098_amd.inputs import load_config
    model = load_config(config)["model"]
    seen, real = [], cf.cf_attn_prompt
    monkeypatch.setattr(cf, "cf_attn_prompt",
                        lambda q, k, v, s, **kw: seen.append(np.diff(s.cpu().numpy())) or real(q, k, v, s, **kw))
    rows = A.profile(config, batch=16, layers=1, decode_steps=1, n_req=100, seed=seed)
    host = cf.cf_trace_gen(cf.model_desc(model), [seed], 100)[0].to_numpy()
    runs = np.array([component in t["comps"] for t in model["types"]])
    ids = np.flatnonzero(runs[host["type"]] & (host["patches"] > 0))[:16]
    n = host["n_img"][ids].astype(int)
    lo, hi = model["patches_per_image"]
    assert len(seen[0]) == n.sum() and seen[0].min() >= lo and seen[0].max() <= hi
    ends = np.cumsum(n)
    sums = [seen[0][b - k:b].sum() for b, k in zip(ends, n)]
    assert sums == host["patches"][ids].astype(int).tolist()
    row = [r for r in rows if r["component"] == component][0]
    assert row["requests"] == 16 and row["tokens"] == sum(sums)
