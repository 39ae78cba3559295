"""The page bookkeeping at the ends of its ranges."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def cf():
    from paper_2512_14098_amd import cf as _cf
    return _cf


def test_map_of_as_many_tokens_as_an_int_counts(cf):
    """n_tok = 2^31 - 1, nearly all of them tokens of no request."""
    n_tok = 2 ** 31 - 1
    print("map of", n_tok, flush=True)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table = i32([[3, -1, -1]])
    q_start, kv_len, slots, pos, head, status = cf.cf_kv_map(i32([5]), i32([40]), table, 16, i32([9, 7, 8]), i32([0]),
                                                            n_tok)
    assert q_start.tolist() == [0, 40] and kv_len.tolist() == [45] and head.tolist() == [2] and status.tolist() == [0]
    assert table.tolist() == [[3, 9, 7]]
    want = [(3, 9, 7)[p // 16] * 16 + p % 16 for p in range(5, 45)]
    assert slots[:40].tolist() == want and pos[:40].tolist() == list(range(5, 45))
    for a in range(40, n_tok, 1 << 28):
        b = min(n_tok, a + (1 << 28))
        assert bool((slots[a:b] == -1).all()) and bool((pos[a:b] == 0).all()), a
