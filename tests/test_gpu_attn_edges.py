"""Edges of the paged-cache calls against plain 64-bit forms: what rows must not see."""
import numpy as np
import pytest

from tests.test_gpu_attn import DT, _i32, _paged_case, _run_paged, _sampled, _say, _want_paged, _want_prompt

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def cf():
    from paper_2512_14098_amd import cf as _cf
    return _cf


# ------------------------------------------------------------------ infinities and NaN of later tokens
def _only_last_row(got, want, n, col):
    """All rows but the last are within their bounds; of the last only column ``col`` is not finite."""
    got = got.double().cpu().numpy()
    out, _, tol, _ = want
    hit = np.zeros(got.shape, bool)
    hit[n - 1, :, col] = True
    assert not np.isfinite(got[hit]).any()
    bad = ~(np.abs(got - out) <= tol) & ~hit
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist())


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("kind,heads,dim,ctx,new", [("bf16", 128, 64, 40, 5), ("fp16", 128, 128, 100, 3),
                                                    ("bf16", 160, 72, 9, 4), ("fp16", 136, 256, 50, 2),
                                                    ("bf16", 128, 64, 6000, 2)])
def test_last_value_is_hidden_where_a_tile_has_one_token(cf, kind, heads, dim, ctx, new, value):
    """As many heads on one key/value head as a workgroup has rows: all rows of a tile see the same
    keys, and the tile's last keys are seen by none of them."""
    _say("one token a tile", kind, heads, dim, ctx, new, value)
    c = _paged_case(kind, [ctx], [new], heads, 1, dim, 16)
    want = _want_paged(c, [ctx], [new], dim ** -0.5, kind)
    p = ctx + new - 1
    c["vc"][c["table"][0, p // 16], 0, p % 16, 3] = value
    _only_last_row(_run_paged(cf, c, [new], heads, 1, dim)[0], want, new, 3)


@pytest.mark.parametrize("value", [float("nan"), float("-inf")])
@pytest.mark.parametrize("kind,dim,ctx", [("bf16", 64, 20), ("fp16", 128, 77), ("bf16", 40, 5000)])
def test_last_value_is_hidden_whatever_max_new_says(cf, kind, dim, ctx, value):
    """Three new tokens of 16 heads on one where the bound on new tokens says one: few rows, a
    token a tile."""
    _say("bound too low", kind, dim, ctx, value)
    c = _paged_case(kind, [ctx], [3], 16, 1, dim, 32)
    want = _want_paged(c, [ctx], [3], dim ** -0.5, kind)
    p = ctx + 2
    c["vc"][c["table"][0, p // 32], 0, p % 32, 5] = value
    _only_last_row(_run_paged(cf, c, [3], 16, 1, dim, max_new=1)[0], want, 3, 5)


@pytest.mark.parametrize("kind,heads,dim,n", [("bf16", 128, 64, 70), ("fp16", 128, 128, 7), ("bf16", 144, 16, 33)])
def test_prompt_last_value_is_hidden_where_a_tile_has_one_token(cf, kind, heads, dim, n):
    _say("prompt, one token a tile", kind, heads, dim, n)
    g = torch.Generator(device="cuda").manual_seed(n)
    q, k, v = (torch.randn((n, h, dim), generator=g, device="cuda").to(DT[kind]) for h in (heads, 1, 1))
    want = _want_prompt(q, k, v, [n], [n], True, dim ** -0.5, kind)
    v[n - 1, 0, 2] = float("nan")
    _only_last_row(cf.cf_attn_prompt(q, k, v, _i32([0, n])), want, n, 2)


@pytest.mark.parametrize("paged", [True, False])
def test_last_value_is_hidden_from_256_heads(cf, paged):
    """The same with two wave groups a workgroup: 256 rows, one token a tile."""
    n, ctx, heads, dim = 200, 30 if paged else 0, 256, 72
    _say("256 heads", paged)
    g = torch.Generator(device="cuda").manual_seed(1)
    m = ctx + n
    q, k, v = (torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
               for s in ((n, heads, dim), (m, 1, dim), (m, 1, dim)))
    hs = [0, 101, 255]
    want = _sampled(q, k, v, list(range(n)), [ctx + j + 1 for j in range(n)], hs, dim ** -0.5, "bf16")
    v[m - 1, 0, 7] = float("inf")
    if paged:
        kc, vc = (torch.full((20, 1, 16, dim), float("nan"), device="cuda").to(torch.bfloat16) for _ in range(2))
        cf.cf_kv_write(k, v, kc, vc, torch.arange(m, device="cuda"))
        plan = cf.cf_attn_plan(_i32([0, n]), _i32([m]), n, n, heads, 1, dim)
        out = cf.cf_attn_paged(plan, q, kc, vc, torch.arange(20, dtype=torch.int32, device="cuda")[None])
    else:
        out = cf.cf_attn_prompt(q, k, v, _i32([0, n]))
    _only_last_row(out[:, hs], want, n, 7)
