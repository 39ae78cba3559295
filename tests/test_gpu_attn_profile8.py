"""Rotary positions and the 8-bit cache together, as an executor's iterations use them."""
import numpy as np
import pytest

from tests import attn_ref, kv8_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("rope,cache8", [(None, True), (10000.0, True), (500.0, False)])
def test_iterations_against_plain_attention(rope, cache8):
    """A prefill and three decode steps of one executor, prompts that end inside pages: each step's output is
    that of plain attention over everything written so far, as it is turned and held; the
    hand-over gives what is held."""
    from paper_2512_14098_amd import cf
    from paper_2512_14098_amd.attn_profile import PagedExecutor
    lens, steps, heads, kv_heads, dim = [37, 1, 64, 130], 3, 4, 2, 64
    torch.manual_seed(0)
    ex = PagedExecutor(len(lens), max(lens) + steps + 1, 2, heads, kv_heads, dim, rope=rope, cache8=cache8)
    ctx = torch.zeros(4, dtype=torch.int32, device="cuda")
    new = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ks, vs, have = [[] for _ in lens], [[] for _ in lens], [0] * 4
    for step in range(steps + 1):
        m = lens if step == 0 else [1] * 4
        ex.qkv = torch.randn((sum(m), heads + 2 * kv_heads, dim), device="cuda").to(torch.bfloat16)
        out, status = ex.step(ctx, new, sum(m), max(m))
        assert int(status.sum()) == 0
        q, k, v = ex.qkv[:, :heads], ex.qkv[:, heads:heads + kv_heads], ex.qkv[:, heads + kv_heads:]
        if rope is not None:
            pos = np.concatenate([c + np.arange(n) for c, n in zip(have, m)]).astype(np.int32)
            q, k = cf.cf_rope(q, k, torch.from_numpy(pos).cuda(), ex.freq)
        q, k, v = (t.double().cpu().numpy() for t in (q, k, v))
        if cache8:
            k, v = ref.held(*ref.quantise(k, "bf16")), ref.held(*ref.quantise(v, "bf16"))
        at = 0
        for i, c in enumerate(m):
            ks[i].append(k[at:at + c])
            vs[i].append(v[at:at + c])
            have[i] += c
            kk, vv = np.concatenate(ks[i]), np.concatenate(vs[i])
            want, _, tol, _ = attn_ref.attend(q[at:at + c], kk, vv, [len(kk) - c + j + 1 for j in range(c)], dim ** -0.5,
                                              "bf16")
            assert np.all(np.abs(out[at:at + c].double().cpu().numpy() - want) <= tol), (step, i)
            at += c
        ctx = ctx + new
        new = torch.ones_like(new)
    if cache8:
        k, v, start = ex.hand_over(ctx, sum(have))
        assert start.cpu().tolist() == np.concatenate([[0], np.cumsum(have)]).tolist()
        for got, want in ((k, ks), (v, vs)):
            assert np.array_equal(got.double().cpu().numpy(), np.concatenate([np.concatenate(w) for w in want]))


def test_profile_of_c1():
    from paper_2512_14098_amd import attn_profile
    rows = attn_profile.profile("c1", batch=16, layers=2, decode_steps=2, n_req=200, rope=10000.0, cache8=True)
    assert [r["step"] for r in rows] == ["prefill", "hand over", "decode 0", "decode 1", "encode"]
    assert all(r["requests"] == 16 and r["attention_s"] > 0 for r in rows)
    assert rows[3]["tokens"] == rows[0]["tokens"] + 32
