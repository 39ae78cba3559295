"""The paged-cache calls together, as an executor's iterations make them."""
import numpy as np
import pytest

from tests import attn_ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_profile_of_c1_and_c2():
    from paper_2512_14098_amd import attn_profile
    for config, encoders in (("c1", ["E"]), ("c2", ["E_img", "E_aud"])):
        rows = attn_profile.profile(config, batch=16, layers=2, decode_steps=2, n_req=200)
        assert [r["step"] for r in rows] == ["prefill", "decode 0", "decode 1"] + ["encode"] * len(encoders)
        assert [r["component"] for r in rows[3:]] == encoders
        assert all(r["requests"] == 16 and r["attention_s"] > 0 and r["model_s"] > 0 for r in rows)
        assert rows[2]["tokens"] == rows[0]["tokens"] + 32


def test_iterations_against_plain_attention():
    """A prefill and three decode steps of one executor: each step's output is that of plain
    attention over everything written so far, through pages the map handed out."""
    from paper_2512_14098_amd.attn_profile import PagedExecutor
    lens, steps, heads, kv_heads, dim = [37, 1, 64, 130], 3, 4, 2, 64
    torch.manual_seed(0)
    ex = PagedExecutor(len(lens), max(lens) + steps + 1, 1, heads, kv_heads, dim)
    ctx = torch.zeros(4, dtype=torch.int32, device="cuda")
    new = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ks, vs = [[] for _ in lens], [[] for _ in lens]
    for step in range(steps + 1):
        m = lens if step == 0 else [1] * 4
        ex.qkv = torch.randn((sum(m), heads + 2 * kv_heads, dim), device="cuda").to(torch.bfloat16)
        out, status = ex.step(ctx, new, sum(m), max(m))
        assert int(status.sum()) == 0
        at = 0
        for i, c in enumerate(m):
            x = ex.qkv[at:at + c].float().cpu().numpy()
            ks[i].append(x[:, heads:heads + kv_heads])
            vs[i].append(x[:, heads + kv_heads:])
            k, v = np.concatenate(ks[i]), np.concatenate(vs[i])
            want, _, tol, _ = attn_ref.attend(x[:, :heads], k, v, [len(k) - c + j + 1 for j in range(c)], dim ** -0.5,
                                              "bf16")
            got = out[at:at + c].double().cpu().numpy()
            assert np.all(np.abs(got - want) <= tol), (step, i)
            at += c
        ctx = ctx + new
        new = torch.ones_like(new)
    assert int(ex.head) == sum(-(-(c + steps) // ex.page) for c in lens)
