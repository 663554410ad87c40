"""conf_kv_attend_pages and conf_kv_load_pages against the formulas in 64 bits.

Tolerance of the attention's outputs, from the arithmetic: every probability is rounded to fp16 once as an operand (2^-11 of it) and
so is the result; a score is a float32 sum of D products, off by at most (D + 4) 2^-24 of sum |q_d K_d| * sm, which moves a
probability by twice that, relative; exponentials, sums and weights of the merges stay under 2^-18 together.  Operands
hold probabilities lifted so that a row's largest is 2^4.5 or more where half a step of the smallest fp16 numbers is 2^-25, so
that n of them are off by n 2^-29 of the largest value.  A difference of two maps has both maps' errors, the second's times its
weight."""
import math

import numpy as np
import pytest

from oracle import confkv_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch


def _handle(lib, B, G, H, D, max_paged, **kw):
    return lib.ConfKV(**dict(dict(n_layers=1, batch=B, n_q_heads=G * H, n_kv_heads=H, head_dim=D, vocab=100, capacity=64, fp16_window=16,
                                  protected_window=16, n_tight=[32], n_loose=[32], max_paged=max_paged), **kw))


def _reference(q, k, v, first, sm, lam=None):
    """Queries [n][G][D] of one kv-head at positions first .. over rows k, v: (out, tolerance); lam [n][G / 2]."""
    n, G, D = q.shape
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    s = np.einsum("tgd,kd->tgk", q, k) * sm
    size = np.einsum("tgd,kd->tgk", np.abs(q), np.abs(k)).max(-1, keepdims=True) * sm * (D + 4) * 2.0 ** -24
    s = np.where(np.arange(len(k)) > first + np.arange(n)[:, None, None], -np.inf, s)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    # (over the rows that a query sees: a weight of zero does not silence a value that is no number)
    over = lambda x: np.stack([p[t, :, :first + t + 1] @ x[:first + t + 1] for t in range(n)])
    o = over(v)
    tol = (2.0 ** -11 + 2.0 ** -18 + 2 * size) * over(np.abs(v)) + len(k) * 2.0 ** -29 * np.abs(v[np.isfinite(v)]).max()
    if lam is not None:
        l = lam.astype(np.float64)[..., None]
        o, tol = o[:, 0::2] - l * o[:, 1::2], tol[:, 0::2] + np.abs(l) * tol[:, 1::2]
    return o, tol + 2.0 ** -11 * np.abs(o) + 2.0 ** -25


class _Case:
    """Pages full of NaN where no token is, rows full of a mark where no sequence is."""
    MARK = 777.0

    def __init__(self, lib, torch, D, G, H, page, new, context, heads_first=False, diff=False, gap=3, seed=0, spread=1.0, room=0,
                 own_rows=True):
        self.torch, self.D, self.G, self.H, self.page, self.new, self.context = torch, D, G, H, page, list(new), list(context)
        self.B, self.rng, self.diff = len(new), np.random.default_rng(seed), diff
        lens = [a + b for a, b in zip(new, context)]
        counts = [-(-n // page) for n in lens]
        self.wide = max(1, max(counts)) + room
        self.n_pages = sum(counts) + 2
        ids = self.rng.permutation(self.n_pages)
        self.table, at = np.full((self.B, self.wide), -7, np.int32), 0
        for b, m in enumerate(counts):
            self.table[b, :m] = ids[at:at + m]
            at += m
        self.pools = [np.full((self.n_pages, page, H, D), np.nan, np.float16) for _ in range(2)]
        self.k, self.v = [], []
        for b in range(self.B):
            self.k.append(self.normal(lens[b], H, D, scale=spread))
            self.v.append(self.normal(lens[b], H, D))
        self.starts, r = [], gap
        for n in new:
            self.starts.append(r)
            r += n + gap
        self.R = r
        self.q = self.normal(self.R, G * H, D)
        self.lam = self.rng.uniform(-0.5, 1.5, (self.R, G * H // 2)).astype(np.float32) if diff else None
        self.kv = _handle(lib, self.B, G, H, D, self.wide * page)
        self.heads_first, self.own_rows = heads_first, own_rows
        self.upload()

    def normal(self, *shape, scale=1.0):
        return (scale * self.rng.standard_normal(shape)).astype(np.float16)

    def on(self, x):
        return self.torch.from_numpy(np.ascontiguousarray(x)).cuda()

    def upload(self):
        """Pools with the earlier tokens (all tokens without rows of their own), row tensors with the new ones."""
        rows = [np.full((self.R, self.H, self.D), np.nan, np.float16) for _ in range(2)]
        for pool, row, x in zip(self.pools, rows, (self.k, self.v)):
            pool[:] = np.nan
            for b in range(self.B):
                self.place(pool, b, x[b], self.context[b] if self.own_rows else len(x[b]))
                row[self.starts[b]:self.starts[b] + self.new[b]] = x[b][self.context[b]:]
        self.pages = [self.on(p.transpose(0, 2, 1, 3)).transpose(1, 2) if self.heads_first else self.on(p) for p in self.pools]
        self.rows = [self.on(r) if self.own_rows else None for r in rows]

    def place(self, pool, b, x, n):
        for t in range(n):
            pool[self.table[b, t // self.page], t % self.page] = x[t]

    def call(self, **kw):
        torch, i32 = self.torch, np.int32
        self.out = torch.full((self.R, self.G * self.H // (2 if self.diff else 1), self.D), self.MARK, dtype=torch.float16, device="cuda")
        args = dict(tokens=max(self.new), starts=self.on(np.array(self.starts, i32)), new=self.on(np.array(self.new, i32)),
                    lam=None if self.lam is None else self.on(self.lam))
        self.kv.attend_pages(self.on(self.q), *self.rows, self.out, *self.pages, self.on(self.table),
                             self.on(np.array(self.context, i32)), **dict(args, **kw))

    def references(self):
        for b, (n, c, s) in enumerate(zip(self.new, self.context, self.starts)):
            for g in range(self.H if n else 0):
                G = self.G
                lam = None if self.lam is None else self.lam[s:s + n, g * G // 2:(g + 1) * G // 2]
                yield b, g, s, n, _reference(self.q[s:s + n, g * G:(g + 1) * G], self.k[b][:, g], self.v[b][:, g], c,
                                             float(np.float32(1 / math.sqrt(self.D))), lam)

    def check(self):
        got, J, worst = self.out.cpu().numpy().astype(np.float64), self.G // (2 if self.diff else 1), 0.0
        claimed = np.zeros(self.R, bool)
        for b, g, s, n, (ref, tol) in self.references():
            claimed[s:s + n] = True
            err = np.abs(got[s:s + n, g * J:(g + 1) * J] - ref) / tol
            assert np.all(err <= 1.0), f"sequence {b} head {g}: off by {np.nanmax(err):.3g} x tolerance at {np.argwhere(~(err <= 1))[:3]}"
            worst = max(worst, float(err.max()))
        assert np.all(got[~claimed] == self.MARK), "rows of no sequence were written"
        for pool, page, x in zip(self.pools, self.pages, (self.k, self.v)):
            for b in range(self.B):
                self.place(pool, b, x[b], len(x[b]))
            assert np.array_equal(page.cpu().numpy().view(np.uint16), pool.view(np.uint16)), "pages"
        return worst

    def run(self, **kw):
        self.call(**kw)
        worst = self.check()
        print(f"worst {worst:.3f} x tolerance", flush=True)
        self.kv.close()


_SHAPES = [
    # D, G, H, page, new, context
    (128, 4, 1, 16, [1], [0]),                              # a sequence's very first token
    (128, 4, 2, 16, [1], [100]),
    (128, 1, 3, 8, [1, 1], [31, 32]),
    (128, 8, 2, 64, [4, 1, 0, 3], [255, 0, 9, 64]),         # 32 rows: the most of the kernel for few
    (128, 16, 1, 32, [2, 1], [1500, 3000]),                 # parts
    (128, 5, 2, 1024, [1, 2], [700, 2500]),
    (64, 4, 3, 16, [1, 1, 1], [0, 513, 2047]),
    (64, 1, 12, 8, [1], [1]),
    (64, 8, 1, 16, [4], [4096]),
    (128, 4, 2, 16, [9], [0]),                              # 36 rows: the kernel for many
    (128, 4, 1, 16, [33, 1, 0, 64], [0, 127, 5, 128]),
    (128, 4, 2, 32, [32, 31], [96, 97]),
    (128, 1, 2, 64, [300], [0]),
    (128, 1, 1, 8, [129, 128, 127], [1, 0, 63]),
    (128, 7, 1, 16, [61], [1000]),                          # parts of it
    (128, 16, 2, 256, [40, 3], [511, 200]),
    (128, 12, 1, 16, [50], [2049]),
    (64, 1, 3, 16, [333, 1], [0, 333]),
    (64, 4, 2, 16, [65, 66], [63, 0]),
    (64, 8, 1, 128, [100], [5000]),
]


@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("D,G,H,page,new,context", _SHAPES)
def test_chunks_of_all_lengths(lib, torch_cuda, D, G, H, page, new, context, heads_first):
    _Case(lib, torch_cuda, D, G, H, page, new, context, heads_first=heads_first, room=2 * heads_first).run()


@pytest.mark.parametrize("D,G,H,page,new,context", [
    (128, 2, 2, 16, [1, 1], [0, 300]), (128, 4, 1, 16, [1], [3000]), (64, 6, 2, 8, [1, 3], [50, 0]), (128, 16, 1, 16, [1], [10]),
    (128, 4, 2, 32, [70, 5], [0, 700]), (128, 2, 1, 16, [200], [100]), (64, 2, 3, 64, [90], [3000]), (128, 12, 1, 16, [30], [0]),
])
def test_differences_of_two_maps(lib, torch_cuda, D, G, H, page, new, context):
    _Case(lib, torch_cuda, D, G, H, page, new, context, diff=True).run()


@pytest.mark.parametrize("new,context", [([1, 1], [40, 700]), ([50, 20], [3, 600])])
def test_new_tokens_that_the_pages_hold_already(lib, torch_cuda, new, context):
    _Case(lib, torch_cuda, 128, 4, 2, 16, new, context, own_rows=False).run()


def test_large_scores(lib, torch_cuda):
    """Scores of some hundreds: the running reference moves often and by much."""
    _Case(lib, torch_cuda, 128, 4, 1, 16, [40], [900], spread=12.0).run()
    _Case(lib, torch_cuda, 128, 4, 1, 16, [2], [900], spread=12.0).run()


def test_calls_without_new_tokens(lib, torch_cuda):
    """Nobody has any, no rows, no tokens: nothing is written."""
    for n in (0, 3):
        c = _Case(lib, torch_cuda, 128, 4, 2, 16, [n, 0], [30, 7])
        c.new = [0, 0]
        before = [p.clone() for p in c.pages]
        for tokens in (1, 3, 50, 0):
            c.call(tokens=tokens)
            assert (c.out == c.MARK).all()
        assert all(torch_cuda.equal(a.view(torch_cuda.int16), b.view(torch_cuda.int16)) for a, b in zip(before, c.pages))
        c.kv.close()
    kv = _handle(lib, 1, 4, 2, 128, 64)
    t = lambda *s: torch_cuda.zeros(s, dtype=torch_cuda.float16, device="cuda")
    i32 = torch_cuda.zeros(1, dtype=torch_cuda.int32, device="cuda")
    kv.attend_pages(t(0, 8, 128), t(0, 2, 128), t(0, 2, 128), t(0, 8, 128), t(4, 16, 2, 128), t(4, 16, 2, 128), i32.reshape(1, 1), i32, tokens=4,
                    starts=i32)
    kv.close()


@pytest.mark.parametrize("T", [1, 30])
def test_rows_of_padded_batches(lib, torch_cuda, T):
    """[B][T] rows of which every sequence uses its first ones; weights for all rows at once; one kv-head, one page."""
    torch, B, wide = torch_cuda, 3, T + 2
    new = [T, max(0, T - 1), min(T, 2)]
    c = _Case(lib, torch, 128, 2, 1, 64, new, [3, 0, 60 - T], diff=True, gap=0)
    q, k, v = (np.full((B, wide) + x.shape[1:], 9.0, np.float16) for x in (c.q, c.k[0], c.v[0]))
    for b, (n, s) in enumerate(zip(new, c.starts)):
        q[b, :n], k[b, :n], v[b, :n] = c.q[s:s + n], c.k[b][c.context[b]:], c.v[b][c.context[b]:]
    c.lam = np.broadcast_to(c.lam[0], c.lam.shape)
    out = torch.full((B, wide, 1, 128), c.MARK, dtype=torch.float16, device="cuda")
    i32 = lambda x: c.on(np.array(x, np.int32))
    pages = [p.as_strided(p.shape, (p.stride(0), p.stride(1), 1, 1)) for p in c.pages]        # (a stride that nothing uses)
    c.kv.attend_pages(c.on(q), c.on(k), c.on(v), out, *pages, c.on(c.table), i32(c.context), tokens=T, starts=i32([b * wide for b in range(B)]),
                      new=i32(new), lam=c.on(c.lam[0]))
    c.out = torch.full((c.R, 1, 128), c.MARK, dtype=torch.float16, device="cuda")
    for b, (n, s) in enumerate(zip(new, c.starts)):
        c.out[s:s + n] = out[b, :n]
        assert (out[b, n:] == c.MARK).all()
    c.check()
    c.kv.close()


def test_more_than_a_wavefront_of_sequences(lib, torch_cuda):
    B = 150
    _Case(lib, torch_cuda, 64, 2, 1, 8, [(1, 0, 2)[b % 3] for b in range(B)], [b % 40 for b in range(B)], gap=0).run()
    _Case(lib, torch_cuda, 64, 4, 1, 8, [(1, 0, 9)[b % 3] for b in range(B)], [7 * b for b in range(B)], gap=1).run()


@pytest.mark.parametrize("T", [1, 3, 40])
def test_equal_lengths_without_starts(lib, torch_cuda, T):
    """[B][T] tensors, every sequence with T new tokens, weights that are the same for all rows."""
    torch = torch_cuda
    c = _Case(lib, torch, 128, 2, 2, 16, [T] * 3, [5, 0, 130], diff=True, gap=0)
    lam = c.lam[0]
    c.lam = np.broadcast_to(lam, c.lam.shape)
    shaped = lambda x, h: x.reshape(3, T, h, c.D)
    c.out = torch.full((3 * T, 2, c.D), c.MARK, dtype=torch.float16, device="cuda")
    c.kv.attend_pages(shaped(c.on(c.q), 4), *(shaped(r, 2) for r in c.rows), shaped(c.out, 2), *c.pages, c.on(c.table),
                      c.on(np.array(c.context, np.int32)), lam=c.on(lam))
    c.check()
    c.kv.close()


@pytest.mark.parametrize("new,context", [([1], [70]), ([3], [600]), ([70], [30]), ([64], [700])])
@pytest.mark.parametrize("what", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("plane", ["k", "v"])
def test_values_that_are_no_numbers(lib, torch_cuda, new, context, what, plane):
    """They show in the rows that see their token, and in no other."""
    c = _Case(lib, torch_cuda, 128, 4, 1, 16, new, context)
    for t in (context[0] // 2, context[0] + new[0] // 2):
        getattr(c, plane)[0][t, 0, 5] = what
    c.upload()
    c.call()
    got = c.out.cpu().numpy().astype(np.float64)[c.starts[0]:c.starts[0] + new[0]]
    with np.errstate(all="ignore"):
        (_, _, _, _, (ref, tol)), = c.references()
        fine = np.isfinite(ref)
        tol = np.where(np.isfinite(tol), tol, np.inf)
    if plane == "v":
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        assert np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)])
    else:                                       # a score that is no number, or infinite upwards, leaves none
        assert np.array_equal(np.isnan(got), np.isnan(ref))
    assert np.all(np.abs(got[fine] - ref[fine]) <= tol[fine])
    c.kv.close()


def test_a_value_of_nearly_no_weight_that_is_infinite(lib, torch_cuda):
    """A weight far below fp16's numbers still makes its value's channel infinite."""
    for new in ([1], [40]):
        c = _Case(lib, torch_cuda, 128, 4, 1, 16, new, [200])
        c.q[:] = 4.0
        c.k[0][:] = 0.25
        c.k[0][50] = -0.25
        c.v[0][50, 0, 7] = np.inf
        c.upload()
        c.call()
        got = c.out.cpu().numpy()[c.starts[0]:c.starts[0] + new[0]].astype(np.float64)
        assert np.all(got[:, :, 7] == np.inf) and np.all(np.isfinite(np.delete(got, 7, 2)))
        c.kv.close()


def test_lengths_are_held_within_bounds(lib, torch_cuda):
    """Counts, contexts, starts and table entries from outside reach no memory that is not the call's."""
    torch = torch_cuda
    B, T, H, G, D, page, wide = 6, 40, 1, 4, 128, 16, 4
    kv = _handle(lib, B, G, H, D, wide * page)
    rng = np.random.default_rng(3)
    n = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float16)).cuda()
    R = B * T
    q, k, v, pk, pv = n(R, G * H, D), n(R, H, D), n(R, H, D), n(B * wide, page, H, D), n(B * wide, page, H, D)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table = torch.arange(B * wide, dtype=torch.int32, device="cuda").reshape(B, wide)
    before = pk.clone()
    out = torch.full((R, G * H, D), 777.0, dtype=torch.float16, device="cuda")
    # count below 0 and above T, context below 0 and behind the room, a start outside, rows that end
    new, context, starts = [-3, 99, 5, 5, 5, 40], [0, -9, 1 << 30, 0, 62, 0], [0, T, 2 * T, R + 5, 4 * T, R - 7]
    kv.attend_pages(q, k, v, out, pk, pv, table, i32(context), tokens=T, starts=i32(starts), new=i32(new))
    want = [(0, 0), (T, 0), (0, 64), (0, 0), (2, 62), (7, 0)]
    touched = np.zeros(R, bool)
    same = np.ones((B * wide, page), bool)
    for b, (m, c) in enumerate(want):
        if m == 0:
            continue
        touched[starts[b]:starts[b] + m] = True
        rows = torch.cat([before[b * wide:(b + 1) * wide].reshape(wide * page, H, D)[:c], k[starts[b]:starts[b] + m]])
        flat = pk[b * wide:(b + 1) * wide].reshape(wide * page, H, D)
        assert torch.equal(flat[:c + m], rows)
        same[b * wide:(b + 1) * wide].reshape(-1)[c:c + m] = False
        values = pv[b * wide:(b + 1) * wide].reshape(wide * page, H, D)[:c + m].cpu().numpy()[:, 0]
        ref, tol = _reference(q[starts[b]:starts[b] + m].cpu().numpy(), rows.cpu().numpy()[:, 0], values, c, float(np.float32(1 / math.sqrt(D))))
        assert np.all(np.abs(out[starts[b]:starts[b] + m].cpu().numpy() - ref) <= tol)
    assert np.all((out.cpu().numpy() == 777.0).all((1, 2)) == ~touched)
    assert torch.equal(pk[torch.from_numpy(same).cuda()], before[torch.from_numpy(same).cuda()])
    # entries that are no pages: nothing is written for them, the others get theirs
    pk.copy_(before)
    table[1, 0], table[1, 1] = -1, B * wide
    kv.attend_pages(q, k, v, out, pk, pv, table, i32([0] * B), tokens=T, starts=i32([b * T for b in range(B)]), new=i32([0, 40, 0, 0, 0, 0]))
    assert torch.equal(pk[6].reshape(page, H, D)[:8], k[T + 32:T + 40]) and torch.equal(pk[:4], before[:4]) and torch.equal(pk[8:], before[8:])
    assert torch.equal(pk[4:6], before[4:6])
    kv.close()


def test_planes_that_take_turns(lib, torch_cuda):
    """Keys and values of a page side by side in one tensor."""
    c = _Case(lib, torch_cuda, 128, 4, 2, 16, [20, 1], [30, 99])
    both = c.torch.stack([c.pages[0], c.pages[1]], 1).contiguous()
    c.pages = [both[:, 0], both[:, 1]]
    c.run()


def test_recorded_calls_follow_the_lengths(lib, torch_cuda):
    """A decode loop and chunks, recorded once each with one workspace between them, replayed with lengths that move on."""
    torch = torch_cuda
    B, H, G, D, page, wide = 2, 2, 4, 128, 16, 64
    kv = _handle(lib, B, G, H, D, wide * page)
    eager = _handle(lib, B, G, H, D, wide * page)
    rng = np.random.default_rng(11)
    n = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float16)).cuda()
    pools = [n(B * wide, page, H, D) for _ in range(2)]
    table = torch.randperm(B * wide).int().cuda().reshape(B, wide)
    context, new = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    graphs = {}
    for T in (1, 48):
        q, k, v = n(B, T, G * H, D), n(B, T, H, D), n(B, T, H, D)
        out = torch.zeros(B, T, G * H, D, dtype=torch.float16, device="cuda")
        starts = torch.arange(B, dtype=torch.int32, device="cuda") * T
        call = lambda h, o, p: h.attend_pages(q, k, v, o, *p, table, context, starts=starts, new=new)
        call(kv, out, [x.clone() for x in pools])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(kv, out, pools)
        graphs[T] = (g, q, k, v, out, starts)
    for T, c, m in [(48, (0, 700), (48, 30)), (1, (48, 730), (1, 1)), (1, (49, 731), (0, 1)), (48, (500, 3), (1, 48)), (1, (1000, 0), (1, 1))]:
        g, q, k, v, out, starts = graphs[T]
        q.copy_(n(*q.shape)), k.copy_(n(*k.shape)), v.copy_(n(*v.shape))
        context.copy_(torch.tensor(c, dtype=torch.int32)), new.copy_(torch.tensor(m, dtype=torch.int32))
        other, want = [x.clone() for x in pools], out.clone()
        eager.attend_pages(q, k, v, want, *other, table, context, starts=starts, new=new)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(torch.equal(x, y) for x, y in zip(pools, other))
    kv.close(), eager.close()


def test_results_repeat_to_the_bit(lib, torch_cuda):
    for new, context in (([1, 1], [3000, 40]), ([60], [2000])):
        c = _Case(lib, torch_cuda, 128, 4, 2, 16, new, context)
        c.call()
        first = c.out.clone()
        for _ in range(3):
            c.call()
            assert torch_cuda.equal(first, c.out)
        c.kv.close()


def test_far_pages(lib, torch_cuda):
    """Pages whose offsets pass 32 bits."""
    torch = torch_cuda
    H, G, D, page, n_pages = 2, 4, 128, 64, 150000                  # 2.5e9 values in a plane
    pools = [torch.empty(n_pages, page, H, D, dtype=torch.float16, device="cuda") for _ in range(2)]
    c = _Case(lib, torch, D, G, H, page, [2, 40], [300, 100])
    ids = np.array([n_pages - 1 - 7 * i for i in range(c.n_pages)])
    for pool, small in zip(pools, c.pages):
        pool[torch.from_numpy(ids).cuda()] = small
    c.table = np.where(c.table >= 0, ids[np.clip(c.table, 0, None)], -1).astype(np.int32)
    small, c.pages = c.pages, pools
    c.call()
    c.pages = [pool[torch.from_numpy(ids).cuda()] for pool in pools]
    back = {int(i): j for j, i in enumerate(ids)}
    c.table = np.array([[back.get(int(e), -7) for e in row] for row in c.table], np.int32)
    c.check()
    c.kv.close()


def test_refusals(lib, torch_cuda):
    torch, b = torch_cuda, lib.binding
    B, H, G, D, page = 2, 2, 3, 128, 16
    kv = _handle(lib, B, G, H, D, 4 * page)
    t = lambda *s, d=torch.float16: torch.zeros(s, dtype=d, device="cuda")
    i32 = torch.int32
    ok = dict(q16=t(B, 2, G * H, D), knew16=t(B, 2, H, D), vnew16=t(B, 2, H, D), out16=t(B, 2, G * H, D), pages_k=t(9, page, H, D),
              pages_v=t(9, page, H, D), table=t(B, 4, d=i32), context=t(B, d=i32))
    kv.attend_pages(**ok)
    kv.attend_pages(**dict(ok, knew16=None, vnew16=None))

    def status(**kw):
        with pytest.raises(lib.ConfKVError) as e:
            kv.attend_pages(**dict(ok, **kw))
        return e.value.status
    assert status(table=t(B, 5, d=i32)) == b.ERR_INVALID_ARG                       # more than max_paged
    assert status(knew16=None) == b.ERR_INVALID_ARG
    assert status(out16=ok["q16"]) == b.ERR_INVALID_ARG
    # Tensors that are read and written: the same keys and values, lengths and tables inside the outputs or the pages.
    assert status(pages_v=ok["pages_k"]) == b.ERR_INVALID_ARG
    kv.attend_pages(**dict(ok, pages_v=ok["pages_k"], knew16=None, vnew16=None))
    for place in ("out16", "pages_v"):
        ints = ok[place].view(i32).reshape(-1)
        for name in ("starts", "new", "context"):
            assert status(**{name: ints[1:3]}) == b.ERR_INVALID_ARG
        assert status(table=ints[:8].reshape(2, 4)) == b.ERR_INVALID_ARG
    pairs = _handle(lib, B, 2, H, D, 4 * page)
    for place in ("out", "pages_v"):
        out = t(B, 2, 2, D)
        with pytest.raises(lib.ConfKVError):
            pairs.attend_pages(**dict(ok, q16=t(B, 2, 4, D), out16=out, lam=(out if place == "out" else ok[place]).view(torch.float32).reshape(-1)[2:4]))
    pairs.close()
    for bad in (12, 4):
        assert status(pages_k=t(9, bad, H, D), pages_v=t(9, bad, H, D)) == b.ERR_INVALID_ARG
    once = t(1, page, H, D).expand(9, page, H, D)
    assert status(pages_k=once, pages_v=once) == b.ERR_INVALID_ARG                   # rows that overlap
    odd = t(9, page, H, D + 4)[..., :D]
    assert status(pages_k=odd, pages_v=odd) == b.ERR_INVALID_ARG                     # strides
    inside = t(40, page, H, D)
    assert status(pages_k=inside[:9], pages_v=inside[9:18], knew16=inside[3].reshape(-1)[:B * 2 * H * D].reshape(B, 2, H, D)) == b.ERR_INVALID_ARG
    for name, bad in (("table", t(B, 4)), ("table", t(3, 4, d=i32)), ("context", t(3, d=i32)), ("q16", t(B, 2, G * H, 64)),
                      ("pages_k", t(9, page, H, 64)), ("out16", t(B, 2, G * H - 1, D)), ("starts", t(B)), ("new", t(5, d=i32)),
                      ("knew16", t(B, 3, H, D))):
        with pytest.raises(ValueError):
            kv.attend_pages(**dict(ok, **{name: bad}))
    with pytest.raises(lib.ConfKVError):                                             # an odd group has no pairs
        kv.attend_pages(**dict(ok, lam=t(B, 2, 3, d=torch.float32), out16=t(B, 2, 3, D)))
    none = _handle(lib, B, G, H, D, 0)
    with pytest.raises(lib.ConfKVError) as e:
        none.attend_pages(**ok)
    assert e.value.status == b.ERR_INVALID_ARG
    with pytest.raises(lib.ConfKVError):
        kv.load_pages(0, ok["pages_k"], ok["pages_v"], ok["table"], 65)
    with pytest.raises(lib.ConfKVError) as e:
        kv.load_pages(1, ok["pages_k"], ok["pages_v"], ok["table"], 5)
    assert e.value.status == b.ERR_BAD_LAYER
    with pytest.raises(lib.ConfKVError) as e:
        kv.load_pages(0, ok["pages_k"], ok["pages_v"], ok["table"], 64)
    assert e.value.status == b.ERR_CAPACITY
    kv.close(), none.close()


# ---- a paged prompt becomes the cache ----

@pytest.mark.parametrize("D,scales,layout,W,page,T0", [
    (128, "token", "contiguous", 40, 16, 200), (128, "token", "contiguous", -1, 8, 65), (64, "token", "contiguous", 16, 64, 333),
    (128, "channel", "contiguous", 20, 16, 190), (128, "token", "paged", 16, 32, 250), (128, "token", "contiguous", 40, 16, 0),
    (128, "token", "contiguous", 40, 1024, 1),
])
@pytest.mark.parametrize("heads_first", [False, True])
def test_a_prompt_from_pages_is_the_prompt(lib, torch_cuda, D, scales, layout, W, page, T0, heads_first):
    """The same cache to the bit as conf_kv_load_prefill's of the same rows."""
    torch, B, H, G = torch_cuda, 3, 2, 2
    kw = dict(capacity=512, fp16_window=W, protected_window=16, n_tight=[300], n_loose=[300], scale_mode=scales, layout=layout,
              evict_page=16 if layout == "paged" else 0)
    a, z = (_handle(lib, B, G, H, D, 0, **kw) for _ in range(2))
    rng = np.random.default_rng(T0)
    k, v = (torch.from_numpy(rng.standard_normal((B, H, T0, D)).astype(np.float16)).cuda() for _ in range(2))
    ema = torch.from_numpy(rng.random((B, H, T0)).astype(np.float32)).cuda() if T0 else None
    m = max(1, -(-T0 // page))
    table = torch.from_numpy(rng.permutation(B * m).astype(np.int32)).cuda().reshape(B, m)
    pools = []
    for x in (k, v):
        pool = torch.full((B * m, page, H, D), math.nan, dtype=torch.float16, device="cuda")
        if heads_first:
            pool = pool.transpose(1, 2).contiguous().transpose(1, 2)
        for t in range(T0):
            pool[table[:, t // page].long(), t % page] = x[:, :, t]
        pools.append(pool)
    a.load_prefill(0, k, v, ema)
    z.load_pages(0, *pools, table, T0, ema)
    for b in range(B):
        for g in range(H):
            x, y = a.export(0, b, g), z.export(0, b, g)
            for name in x:
                assert np.array_equal(np.asarray(x[name]).view(np.uint8) if name != "n" else x[name],
                                      np.asarray(y[name]).view(np.uint8) if name != "n" else y[name]), name
    a.close(), z.close()
