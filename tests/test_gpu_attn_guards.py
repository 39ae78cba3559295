"""The paged-cache calls write inside their arrays whatever the device data hold: every array is
the middle of a larger buffer whose ends are compared afterwards."""
import ctypes as C

import numpy as np
import pytest

from tests import attn_ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

EDGE = 1 << 16  # bytes kept on either side
BIG = [-2 ** 31, -2 ** 27, -17, -1, 0, 1, 2, 3, 15, 16, 40, 127, 128, 2 ** 20, 2 ** 27 - 1, 2 ** 27, 2 ** 27 + 1, 2 ** 28,
       2 ** 30 - 1, 2 ** 30, 2 ** 31 - 16, 2 ** 31 - 1]


@pytest.fixture(scope="module")
def cf():
    from paper_2512_14098_amd import cf as _cf
    return _cf


class Guarded:
    """A device array of n bytes between two known ends; it starts as the same pattern."""

    def __init__(self, n, data=None):
        self.n = n
        self.buf = torch.full((2 * EDGE + n,), 0x5A, dtype=torch.uint8, device="cuda")
        if data is not None:
            self.bytes().copy_(data.contiguous().view(-1).view(torch.uint8))

    def bytes(self):
        return self.buf[EDGE:EDGE + self.n]

    def ptr(self):
        return self.buf.data_ptr() + EDGE

    def view(self, dtype):
        return self.bytes().view(dtype)

    def intact(self):
        ends = torch.cat([self.buf[:EDGE], self.buf[EDGE + self.n:]])
        return bool((ends == 0x5A).all())


def _i32(x):
    return torch.as_tensor(np.asarray(x, np.int64).astype(np.int32)).cuda()


class Step:
    """A paged call through the C ABI on guarded arrays."""

    def __init__(self, cf, n_seq, n_tok, max_new, heads, kv_heads, dim, page, columns, n_pages=9, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        bf = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
        self.cf, self.dim, self.heads, self.n_tok, self.columns = cf, dim, heads, n_tok, columns
        self.kc = Guarded(n_pages * kv_heads * page * dim * 2, bf(n_pages, kv_heads, page, dim))
        self.vc = Guarded(n_pages * kv_heads * page * dim * 2, bf(n_pages, kv_heads, page, dim))
        self.q = Guarded(n_tok * heads * dim * 2, bf(n_tok, heads, dim))
        self.table = Guarded(n_seq * columns * 4,
                             torch.randint(-2, n_pages + 2, (n_seq, columns), generator=g, device="cuda").int())
        self.out, self.lse = Guarded(n_tok * heads * dim * 2), Guarded(n_tok * heads * 4)
        self.c = cf.cf_kv_cache(self.kc.ptr(), self.vc.ptr(), n_pages, page, kv_heads, dim, 0)
        self.d = cf.cf_attn_desc()
        self.d.n_seq, self.d.n_tok, self.d.max_new = n_seq, n_tok, max_new
        self.d.n_heads, self.d.n_kv_heads, self.d.head_dim = heads, kv_heads, dim
        need = C.c_uint64(0)
        assert cf.lib().cf_attn_plan_bytes(C.byref(self.d), C.byref(need)) == 0
        self.work = Guarded(need.value)
        self.d.work_dev, self.d.work_bytes = self.work.ptr(), need.value
        self.d.q_start_dev = self.d.kv_len_dev = self.table.ptr()  # replaced by plan()
        self.inputs = [(x, x.buf.clone()) for x in (self.kc, self.vc, self.q, self.table)]

    def plan(self, starts, kv_len):
        self.keep = Guarded(4 * len(starts), _i32(starts)), Guarded(4 * len(kv_len), _i32(kv_len))
        self.d.q_start_dev, self.d.kv_len_dev = (x.ptr() for x in self.keep)
        assert self.cf.lib().cf_attn_plan(C.byref(self.d), self.cf._stream()) == 0

    def run(self):
        assert self.cf.lib().cf_attn_paged(C.byref(self.d), C.byref(self.c), self.table.ptr(), self.columns, self.q.ptr(),
                                           self.heads * self.dim, self.dim, 0.125, self.out.ptr(), self.lse.ptr(),
                                           self.cf._stream()) == 0
        torch.cuda.synchronize()
        assert self.out.intact() and self.lse.intact() and self.work.intact()
        for x, before in self.inputs:
            assert torch.equal(x.buf, before)


SHAPES = [(3, 34, 30, 4, 2, 64, 16, 6), (3, 34, 3, 4, 2, 64, 16, 6), (5, 300, 300, 8, 1, 128, 32, 9),
          (2, 40, 1, 16, 1, 72, 16, 70), (4, 20, 20, 4, 2, 256, 64, 3), (3, 1600, 1600, 32, 1, 96, 16, 40)]


@pytest.mark.parametrize("shape", SHAPES)
def test_malformed_lengths(cf, shape):
    """Starts in any order, lengths of any size, table entries outside the cache."""
    print("malformed", shape, flush=True)
    n, n_tok = shape[0], shape[1]
    rng = np.random.default_rng(n_tok)
    s = Step(cf, *shape)
    for starts, kv in [([n_tok, 3, -9] + [n_tok] * (n - 2), [-1, 7] + [9] * (n - 2)),
                       ([0] * n + [2 ** 31 - 1], [2 ** 31 - 1] * n), ([-2 ** 31] * (n + 1), [5] * n)] + [
                           (rng.choice(BIG, n + 1), rng.choice(BIG, n)) for _ in range(20)]:
        s.plan(starts, kv)
        s.run()


@pytest.mark.parametrize("shape", SHAPES)
def test_workspace_without_a_plan(cf, shape):
    """A workspace that holds no plan: noise, and words that pass some of the checks."""
    print("no plan", shape, flush=True)
    rng = np.random.default_rng(shape[1])
    s = Step(cf, *shape)
    words = s.work.n // 4
    s.run()  # the pattern of the buffer
    for values in (BIG, [0, 1, 2, 3, 2 ** 27, 2 ** 28], [0, 1, 2, 4, 128, 256], None):
        x = rng.integers(-2 ** 31, 2 ** 31, words) if values is None else rng.choice(values, words)
        s.work.bytes().copy_(_i32(x).view(torch.uint8)[:s.work.n])
        s.run()


def test_tokens_of_no_request_and_lengths_past_the_table(cf):
    """Rows that no request owns are left as they were; a length past the table's row counts as the row."""
    s = Step(cf, 3, 60, 60, 4, 2, 64, 16, 4)
    before = s.out.view(torch.int16).view(60, -1).clone(), s.lse.view(torch.int32).view(60, -1).clone()
    s.plan([5, 8, 8, 50], [64, 9, 2 ** 31 - 1])
    s.run()
    for got, was in zip((s.out.view(torch.int16).view(60, -1), s.lse.view(torch.int32).view(60, -1)), before):
        assert torch.equal(got[:5], was[:5]) and torch.equal(got[50:], was[50:])
        assert bool((got[5:50] != was[5:50]).any(1).all())
    first = s.out.bytes().clone(), s.lse.bytes().clone()
    s.plan([5, 8, 8, 50], [64, 9, 64])
    s.run()
    assert torch.equal(first[0], s.out.bytes()) and torch.equal(first[1], s.lse.bytes())


def test_prompt_tokens_of_no_sequence(cf):
    """The packed call leaves rows outside the sequences as they were, and writes nothing else."""
    n_q, heads, dim = 200, 4, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (Guarded(n_q * h * dim * 2, torch.randn((n_q, h, dim), generator=g, device="cuda").to(torch.bfloat16))
               for h in (heads, 2, 2))
    out, lse = Guarded(n_q * heads * dim * 2), Guarded(n_q * heads * 4)
    rng = np.random.default_rng(0)
    for t, starts in enumerate([[20, 60, 160]] + [rng.choice(BIG + [50, 100, 200], 3) for _ in range(20)]):
        p = _i32(starts)
        a = cf.cf_attn_seqs(2, n_q, n_q, heads, 2, dim, 0, t % 2, p.data_ptr(), p.data_ptr(), q.ptr(), k.ptr(), v.ptr(),
                            heads * dim, dim, 2 * dim, dim, 2 * dim, dim)
        was = out.view(torch.int16).view(n_q, -1).clone()
        assert cf.lib().cf_attn_prompt(C.byref(a), 0.125, out.ptr(), lse.ptr(), cf._stream()) == 0
        torch.cuda.synchronize()
        assert out.intact() and lse.intact()
        if t == 0:
            got = out.view(torch.int16).view(n_q, -1)
            assert torch.equal(got[:20], was[:20]) and torch.equal(got[160:], was[160:])
            assert bool((got[20:160] != was[20:160]).any(1).all())


def test_map_and_write(cf):
    """Block tables, slots and caches with lengths, heads and slots of any size."""
    rng = np.random.default_rng(5)
    n, page, columns, n_free = 40, 16, 5, 60
    for n_tok in (0, 1, 700, 2048, 5000):
        for ordinary in (True, False):
            pick = lambda odd: np.where(rng.random(n) < (0.1 if ordinary else 0.7), rng.choice(odd, n),
                                        rng.integers(0, 50, n))
            ctx, new = pick(BIG), pick([-2 ** 31, -17, 2000] if ordinary else BIG)
            head = int(rng.choice([0, 7, 59, 60] if ordinary else BIG))
            table, free = rng.integers(-3, 100, (n, columns)), rng.integers(-3, 100, n_free)
            t = Guarded(n * columns * 4, _i32(table))
            ins = [Guarded(4 * np.size(x), _i32(x)) for x in (ctx, new, free, [head])]
            outs = dict(q_start=Guarded(4 * (n + 1)), kv_len=Guarded(4 * n), slots=Guarded(8 * n_tok), pos=Guarded(4 * n_tok),
                        head=Guarded(4), status=Guarded(4 * n))
            o = {k: x.ptr() for k, x in outs.items()}
            assert cf.lib().cf_kv_map(n, ins[0].ptr(), ins[1].ptr(), page, t.ptr(), columns, ins[2].ptr(), n_free,
                                      ins[3].ptr(), n_tok, o["q_start"], o["kv_len"], o["slots"], o["pos"], o["head"],
                                      o["status"], cf._stream()) == 0
            torch.cuda.synchronize()
            assert t.intact() and all(x.intact() for x in outs.values())
            if ordinary:  # small enough for the sequential form
                want = attn_ref.kv_map(ctx, new, table, page, free, head, n_tok)
                for name, x in outs.items():
                    got = x.view(torch.int64 if name == "slots" else torch.int32).cpu().numpy()
                    assert np.array_equal(got, np.asarray(want[name])), (n_tok, name)
                assert np.array_equal(t.view(torch.int32).cpu().numpy().reshape(n, columns), want["table"])
    heads, dim, n_pages, n_tok = 3, 24, 7, 300
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((n_tok, heads, dim), generator=g, device="cuda").to(torch.float16) for _ in range(2))
    kc, vc = Guarded(n_pages * heads * 16 * dim * 2), Guarded(n_pages * heads * 16 * dim * 2)
    slots = rng.choice([-2 ** 63, -2 ** 32, -1, n_pages * 16, n_pages * 16 + 1, 2 ** 31, 2 ** 32, 2 ** 63 - 1], n_tok)
    slots[::9] = np.arange(len(slots[::9]))
    sl = torch.as_tensor(slots).cuda()
    c = cf.cf_kv_cache(kc.ptr(), vc.ptr(), n_pages, 16, heads, dim, 1)
    assert cf.lib().cf_kv_write(C.byref(c), n_tok, k.data_ptr(), heads * dim, dim, v.data_ptr(), heads * dim, dim,
                                sl.data_ptr(), cf._stream()) == 0
    torch.cuda.synchronize()
    for x, src in ((kc, k), (vc, v)):
        assert x.intact()
        want = torch.full((n_pages, heads, 16, dim), 0x5A5A, dtype=torch.int16, device="cuda")
        for i, t in enumerate(range(0, n_tok, 9)):
            want[i // 16, :, i % 16] = src[t].view(torch.int16)
        assert torch.equal(x.view(torch.int16), want.view(-1))
