"""Which contexts of many-row requests a plan splits."""
import numpy as np
import pytest

from tests.test_gpu_attn import _compare, _say
from tests.test_gpu_attn_join import Caches

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def cf():
    from paper_2512_14098_amd import cf as _cf
    return _cf


def _split_tiles(cf, lens, new, heads, kv_heads, dim):
    start = torch.tensor([0] + new, device="cuda").cumsum(0).int()
    plan = cf.cf_attn_plan(start, torch.tensor(lens, dtype=torch.int32, device="cuda"), sum(new), max(new), heads, kv_heads, dim)
    return int(plan.work[16:20].view(torch.int32))  # the header's count


@pytest.mark.parametrize("lens,new,heads,kv_heads,dim", [
    ([200], [200], 32, 8, 128), ([170], [20], 32, 8, 128), ([214] * 4, [64] * 4, 32, 8, 128), ([500], [500], 32, 8, 128),
    ([1500] * 15 + [200], [1] * 15 + [200], 32, 8, 128), ([200], [200], 16, 4, 64), ([900] * 4, [500] * 4, 16, 4, 64),
    ([1000], [1000], 32, 8, 96), ([600] * 4, [200] * 4, 32, 8, 96), ([200], [200], 16, 8, 256), ([400], [400], 16, 16, 256), ([214] * 4, [64] * 4, 16, 8, 256)])
def test_whole_where_the_join_costs_more(cf, lens, new, heads, kv_heads, dim):
    """A join takes about as long as 250 keys (50 above 128 columns), storing and reading the parts more where they
    fill the card: contexts that gain less stay whole."""
    assert _split_tiles(cf, lens, new, heads, kv_heads, dim) == 0


@pytest.mark.parametrize("lens,new,heads,kv_heads,dim", [
    ([1040], [40], 32, 8, 128), ([30005] * 3, [5] * 3, 32, 8, 128), ([1220] * 4, [20] * 4, 32, 8, 128),
    ([10100] * 2, [100] * 2, 32, 8, 128), ([2520], [20], 16, 8, 256), ([8200], [200], 8, 1, 128), ([20500], [500], 16, 2, 64)])
def test_split_where_one_round_leaves_the_card_empty(cf, lens, new, heads, kv_heads, dim):
    assert _split_tiles(cf, lens, new, heads, kv_heads, dim) > 0


def test_parts_of_tiles_with_few_rows(cf):
    """Their results cost little: two parts for each workgroup that runs at a time (64 for each of 8 heads), not one:
    90,015 keys in parts of an even share of 704, up to a multiple of 128."""
    start = torch.tensor([0, 5, 10, 15], dtype=torch.int32, device="cuda")
    plan = cf.cf_attn_plan(start, torch.full((3,), 30005, dtype=torch.int32, device="cuda"), 15, 5, 32, 8, 128)
    assert int(plan.work[4:8].view(torch.int32)) == 3 * -(-30005 // 768)  # the header's count of the many-row kernel's items


@pytest.mark.parametrize("width", [16, 8])
@pytest.mark.parametrize("n,busy,many", [(250, 20, 3), (255, 3, 40), (2600, 30, 5), (2600, 700, 9)])
def test_plans_in_order_and_sorted(cf, width, n, busy, many):
    """Requests that wait, with one new token and with many in any order, in one and in three rounds of the plan's
    workgroup; 700 with few rows are sorted by length, fewer are not."""
    _say("order", width, n, busy, many)
    rng = np.random.default_rng(n + busy)
    new = np.zeros(n, int)
    at = rng.permutation(n)
    new[at[:busy]] = rng.integers(1, 5, busy)
    new[at[busy:busy + many]] = rng.integers(10, 60, many)
    lens = np.maximum(new, np.where(new > 0, rng.integers(1, 300, n), rng.integers(1, 20, n)))
    c = Caches(cf, "bf16", lens.tolist(), new.tolist(), 4, 1, 64)
    _compare(*c.run(width, c.plan()), c.want("bf16"))
