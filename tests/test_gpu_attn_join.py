"""Split contexts of many rows, joined by workgroups of the few-row kernel, over caches of either width."""
import numpy as np
import pytest

from tests import attn_ref, kv8_ref as ref
from tests.test_gpu_attn import DT, _compare, _i32, _sampled, _say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def cf():
    from paper_2512_14098_amd import cf as _cf
    return _cf


def _held(x):
    """Rows [tokens][heads][dim] as an 8-bit cache holds them, in their own type."""
    kind = "bf16" if x.dtype == torch.bfloat16 else "fp16"
    return torch.from_numpy(ref.held(*ref.quantise(x.double().cpu().numpy(), kind))).to(x.dtype).cuda()


class Caches:
    """A 16-bit and an 8-bit cache of the same values, written through the calls; page 16."""

    def __init__(self, cf, kind, lens, new, heads, kv_heads, dim, seed=0):
        self.cf, self.new, self.lens, self.args = cf, new, lens, (heads, kv_heads, dim)
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(DT[kind])
        pages = [-(-x // 16) for x in lens]
        order = torch.randperm(sum(pages), generator=g, device="cuda").int()
        self.table = torch.full((len(lens), max(pages)), -1, dtype=torch.int32, device="cuda")
        shape = (sum(pages), kv_heads, 16, dim)
        self.c16 = [torch.zeros(shape, dtype=DT[kind], device="cuda") for _ in range(2)]
        self.c8 = [torch.zeros(shape, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
        self.c8.append(torch.zeros((shape[0], kv_heads, 2, 16), dtype=torch.uint8, device="cuda"))
        self.ks, self.vs, at = [], [], 0
        for i, (x, p) in enumerate(zip(lens, pages)):
            self.table[i, :p] = order[at:at + p]
            at += p
            k, v = _held(rand(x, kv_heads, dim)), _held(rand(x, kv_heads, dim))
            t = torch.arange(x, device="cuda")
            slots = self.table[i, t // 16].long() * 16 + t % 16
            cf.cf_kv_write(k, v, *self.c16, slots)
            cf.cf_kv_write8(k, v, *self.c8, slots)
            self.ks.append(k)
            self.vs.append(v)
        self.q = rand(sum(new), heads, dim)
        self.starts, self.kv = _i32(np.concatenate([[0], np.cumsum(new)])), _i32(lens)

    def plan(self):
        return self.cf.cf_attn_plan(self.starts, self.kv, sum(self.new), max(self.new), *self.args)

    def run(self, width, plan, lse=True):
        if width == 16:
            return self.cf.cf_attn_paged(plan, self.q, *self.c16, self.table, lse=lse)
        return self.cf.cf_attn_paged8(plan, self.q, *self.c8, self.table, lse=lse)

    def want(self, kind):
        parts, at = [], 0
        for i, m in enumerate(self.new):
            f = lambda t: t.float().cpu().numpy()
            parts.append(attn_ref.attend(f(self.q[at:at + m]), f(self.ks[i]), f(self.vs[i]),
                                         [self.lens[i] - m + j + 1 for j in range(m)], self.args[2] ** -0.5, kind))
            at += m
        return [np.concatenate(p) for p in zip(*parts)]


@pytest.mark.parametrize("width", [16, 8])
@pytest.mark.parametrize("kind,heads,kv_heads,dim", [("bf16", 4, 1, 64), ("fp16", 6, 2, 128), ("bf16", 3, 1, 96),
                                                     ("fp16", 2, 1, 256), ("bf16", 5, 1, 16)])
@pytest.mark.parametrize("lens,new", [([9000], [40]), ([9000, 51, 700, 3], [40, 1, 0, 2]), ([700, 900], [90, 300]),
                                      ([20000], [7]), ([260, 129, 130], [64, 70, 129])])
def test_joined(cf, width, kind, heads, kv_heads, dim, lens, new):
    """Alone, among few-row requests and ones that wait, short and long; the same on every call."""
    _say("joined", width, kind, heads, kv_heads, dim, lens, new)
    c = Caches(cf, kind, lens, new, heads, kv_heads, dim)
    plan = c.plan()
    a, b = c.run(width, plan), c.run(width, plan)
    _compare(*a, c.want(kind))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(c.run(width, plan, lse=False), a[0])


@pytest.mark.parametrize("width", [16, 8])
def test_joined_tiles_of_two_groups(cf, width):
    """Tiles of 256 rows: 800 tokens of 64 heads on 2, 60,000 keys."""
    c = Caches(cf, "bf16", [60000], [800], 64, 2, 128)
    rows, hs = [0, 1, 255, 256, 511, 799], [0, 33, 63]
    plan = c.plan()
    assert int(plan.work[16:20].view(torch.int32)) > 0  # the header's count of split tiles
    got = c.run(width, plan)
    want = _sampled(c.q, c.ks[0], c.vs[0], rows, [59200 + j + 1 for j in range(800)], hs, 128 ** -0.5, "bf16")
    _compare(*[x[rows][:, hs] for x in got], want)


@pytest.mark.parametrize("width", [16, 8])
def test_joined_in_a_graph(cf, width):
    """Plan and call captured once, replayed as lengths and queries change, beside eager calls."""
    c = Caches(cf, "bf16", [5000, 2000, 40], [40, 33, 1], 4, 2, 128)

    def step():
        return c.run(width, c.plan())

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse = step()
    for i in range(4):
        c.q.add_(0.25)
        c.kv.copy_(_i32([5000 - 900 * i, 2000 - 10 * i, 40 - i]))
        g.replay()
        torch.cuda.synchronize()
        want, wl = step()
        assert torch.equal(out, want) and torch.equal(lse, wl)


@pytest.mark.parametrize("width", [16, 8])
def test_joined_rows_that_see_little(cf, width):
    """Fewer keys than new tokens, and none at all: zero rows and lse -inf past a split."""
    c = Caches(cf, "bf16", [600, 300], [400, 100], 4, 1, 64)
    c.kv = _i32([390, 0])
    out, lse = c.run(width, c.plan())
    f = lambda t: t.float().cpu().numpy()
    parts = [attn_ref.attend(f(c.q[:400]), f(c.ks[0]), f(c.vs[0]), [j - 9 for j in range(400)], 0.125, "bf16"),
             attn_ref.attend(f(c.q[400:]), f(c.ks[1]), f(c.vs[1]), [0] * 100, 0.125, "bf16")]
    _compare(out, lse, [np.concatenate(p) for p in zip(*parts)])
