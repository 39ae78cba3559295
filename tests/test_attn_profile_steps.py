"""The attention profile's iterations with the device calls replaced by records (no GPU needed)."""
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2512_14098_amd", "libcf.so")),
                                reason="libcf.so not built")


@pytest.fixture
def calls(monkeypatch):
    """attn_profile on host tensors: what it passes to the device calls is recorded."""
    from paper_2512_14098_amd import attn_profile as A
    rec = dict(prompts=[], writes=[], reads=[])

    def kv_map(ctx, new, table, page, free, head, n_tok):
        n = len(ctx)
        return (torch.zeros(n + 1, dtype=torch.int32), ctx + new, torch.zeros(n_tok, dtype=torch.int64),
                torch.zeros(n_tok, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(n, dtype=torch.int32))

    monkeypatch.setattr(A.cf, "cf_kv_map", kv_map)
    monkeypatch.setattr(A.cf, "cf_attn_plan", lambda *a: None)
    monkeypatch.setattr(A.cf, "cf_kv_write", lambda k, v, kc, vc, s: rec["writes"].append((kc.data_ptr(), vc.data_ptr())))
    monkeypatch.setattr(A.cf, "cf_attn_paged",
                        lambda p, q, kc, vc, t: rec["reads"].append((kc.data_ptr(), vc.data_ptr())) or q)
    monkeypatch.setattr(A.cf, "cf_attn_prompt",
                        lambda q, k, v, s, **kw: rec["prompts"].append(np.diff(s.numpy()).tolist()) or q)
    monkeypatch.setattr(A, "_timed", lambda fn: (fn(), 1.0))
    return A, rec


class _Trace:
    """Audio requests of the omni graph: type 2 asks with speech, type 0 with text alone."""

    def __init__(self, ms):
        n = len(ms) + 1
        self.t = dict(type=np.array([0] + [2] * len(ms)), prompt=np.full(n, 20), out=np.full(n, 5), n_img=np.zeros(n, int),
                      patches=np.zeros(n, int), aud_in_ms=np.array([0] + ms), aud_out_ms=np.full(n, 240))

    def to_numpy(self):
        return self.t


def _profile(A, monkeypatch, ms, **kw):
    monkeypatch.setattr(A.cf, "cf_trace_gen", lambda *a: (_Trace(ms), None))
    return A.profile("c2", layers=2, heads=2, kv_heads=1, dim=8, decode_steps=1, device="cpu", **kw)


def test_audio_is_priced_in_the_components_own_unit(calls, monkeypatch):
    """E_aud costs 0.002 s + 1e-6 s a millisecond, whatever the frames of its attention are."""
    A, _ = calls
    ms = [1000, 4481, 150003]
    row = [r for r in _profile(A, monkeypatch, ms) if r["component"] == "E_aud"][0]
    assert row["requests"] == 3
    assert row["model_s"] == pytest.approx(0.002 + 1e-6 * sum(ms), rel=1e-12)
    row = [r for r in _profile(A, monkeypatch, ms, batch=2) if r["component"] == "E_aud"][0]
    assert row["model_s"] == pytest.approx(0.002 + 1e-6 * sum(ms[:2]), rel=1e-12)


def test_long_audio_is_several_windows(calls, monkeypatch):
    """20 ms a frame, 4096 frames a window, the last one shorter; nothing is cut off."""
    A, rec = calls
    row = [r for r in _profile(A, monkeypatch, [1000, 4481, 150003]) if r["component"] == "E_aud"][0]
    assert rec["prompts"][0] == [50, 225, 4096, 7501 - 4096]
    assert row["tokens"] == 50 + 225 + 7501 and row["requests"] == 3


@pytest.mark.parametrize("layers,tokens,caches", [(6, None, 4), (6, 20, 6), (3, None, 3), (6, 32, 5), (1, 20, 1),
                                                  (6, 1 << 20, 1)])
def test_layers_have_caches_of_their_own(calls, monkeypatch, layers, tokens, caches):
    """A pass over the layers reads caches of twice the last-level cache's bytes before it comes back
    to one, or each layer has its own; a layer reads the cache that it wrote."""
    A, rec = calls
    token = 2 * 3 * 8 * 2  # bytes of keys and values
    monkeypatch.setattr(A, "PASS_BYTES", 160 * token)
    ex = A.PagedExecutor(2, 20, layers, 6, 3, 8, device="cpu", tokens=tokens)  # holds 2 x 2 pages of 16: 64 tokens
    if tokens is None:
        monkeypatch.setattr(A, "PASS_BYTES", 64 * 4 * token)
        ex = A.PagedExecutor(2, 20, layers, 6, 3, 8, device="cpu")
    one = torch.ones(2, dtype=torch.int32)
    for step in range(2):
        del rec["writes"][:], rec["reads"][:]
        ex.step(one * (5 + step), one, 2, 1)
        assert rec["writes"] == rec["reads"] and len(rec["reads"]) == layers
        assert len(set(rec["reads"])) == caches and len(set(rec["reads"][:caches])) == caches
        assert rec["reads"][caches:] == rec["reads"][:layers - caches]


def test_profile_sizes_the_caches_by_the_batchs_tokens(calls, monkeypatch):
    """Every layer of a small batch has its own cache."""
    A, rec = calls
    _profile(A, monkeypatch, [1000, 2000])
    assert len(set(rec["reads"])) == 2
