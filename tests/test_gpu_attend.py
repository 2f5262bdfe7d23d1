"""Attention over the paged cache, with and without shared prefixes, against the formula in 64 bits."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2502_11494_b200 import dart  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
NAN = float("nan")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class Case:
    """Sequences (query rows, own tokens), groups as (sequences, prefix tokens); pages in no order, everything that no row sees
    filled with NaN, table entries that nobody may read far out of range."""

    def __init__(self, Hq, Hk, D, page, dtype, seqs, groups=(), before=0, seed=0, sharp=1.0, gap=0, spare=3, qstride=0):
        g = _gen(seed * 7919 + Hq * 131 + D + page + len(seqs))
        dt = TYPES[dtype]
        self.Hq, self.Hk, self.D, self.page, self.seqs, self.groups, self.before, self.gap = Hq, Hk, D, page, list(seqs), list(groups), before, gap
        lens = [L for _, L in seqs] + [L for _, L in groups]
        need = [(L + page - 1) // page for L in lens]
        total = sum(need) + spare
        order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
        self.k = torch.full((total, Hk, page, D), NAN, dtype=dt, device="cuda")
        self.v = torch.full_like(self.k, NAN)
        tables, at = [], 0
        for part in (need[:len(seqs)], need[len(seqs):]):
            t = torch.full((len(part), max(part + [0]) + 2), 2**30, dtype=torch.int32, device="cuda")
            for i, n in enumerate(part):
                t[i, :n] = order[at:at + n]
                at += n
            tables.append(t)
        self.table, self.ptable = tables
        for t, ls in ((self.table, lens[:len(seqs)]), (self.ptable, lens[len(seqs):])):
            for i, L in enumerate(ls):
                s = torch.arange(L, device="cuda")
                for c, size in ((self.k, sharp), (self.v, 1.0)):
                    x = torch.randn((L, Hk, D), generator=g, device="cuda") * size
                    c[t[i].long()[s // page], :, s % page] = x.to(dt)
        n = gap + sum(a for a, _ in seqs)
        self.n = n + gap
        wide = torch.randn((self.n, Hq + qstride, D), generator=g, device="cuda").to(dt)
        self.q = wide[:, :Hq]
        self.kv_len = torch.tensor([L for _, L in seqs], dtype=torch.int32, device="cuda")
        cu = [gap]
        for a, _ in seqs:
            cu.append(cu[-1] + a)
        self.cu = cu
        self.cu_q = torch.tensor(cu, dtype=torch.int32, device="cuda")
        if all(a == 1 for a, _ in seqs) and gap == 0:
            self.cu_q = None
        self.prefix = None
        if groups:
            cg = [before]
            for a, _ in groups:
                cg.append(cg[-1] + a)
            self.prefix = (self.ptable, torch.tensor([L for _, L in groups], dtype=torch.int32, device="cuda"),
                           torch.tensor(cg, dtype=torch.int32, device="cuda"))
            self.cg = cg
        self.cache = dart.PagedCache(self.k, self.v)

    def tokens(self, c, table, L):
        s = torch.arange(L, device="cuda")
        return c[table.long()[s // self.page], :, s % self.page].double()  # [L, Hk, D]

    def reference(self, scale):
        """out, lse and the bound on out's error, in fp64; rows of no sequence NaN."""
        eps = torch.finfo(self.q.dtype).eps
        out = torch.full((self.n, self.Hq, self.D), NAN, dtype=torch.float64, device="cuda")
        lse = torch.full((self.n, self.Hq), NAN, dtype=torch.float64, device="cuda")
        bound, lbound = torch.zeros_like(out), torch.zeros_like(lse)
        R = self.Hq // self.Hk
        for b, (n, L) in enumerate(self.seqs):
            k, v = self.tokens(self.k, self.table[b], L), self.tokens(self.v, self.table[b], L)
            seen = torch.arange(L, device="cuda")[None, :] <= L - n + torch.arange(n, device="cuda")[:, None]
            for i, (a, Lp) in enumerate(self.groups):
                if self.cg[i] <= b < self.cg[i + 1]:
                    k = torch.cat((self.tokens(self.k, self.ptable[i], Lp), k))
                    v = torch.cat((self.tokens(self.v, self.ptable[i], Lp), v))
                    seen = torch.cat((torch.ones((n, Lp), dtype=torch.bool, device="cuda"), seen), 1)
            x = self.q[self.cu[b]:self.cu[b + 1]].double().view(n, self.Hk, R, self.D)
            s = torch.einsum("nhrd,lhd->hrnl", x, k) * scale
            size = torch.einsum("nhrd,lhd->hrnl", x.abs(), k.abs()) * scale
            s = s.masked_fill(~seen, -math.inf)
            p = torch.softmax(s, -1).nan_to_num(0.0)  # rows that see nothing: zeros
            o = torch.einsum("hrnl,lhd->nhrd", p, v).reshape(n, self.Hq, self.D)
            a = torch.einsum("hrnl,lhd->nhrd", p, v.abs()).reshape(n, self.Hq, self.D)
            rows = slice(self.cu[b], self.cu[b + 1])
            out[rows] = o
            ls = torch.logsumexp(s, -1) if s.shape[-1] else torch.full(s.shape[:-1], -math.inf, dtype=s.dtype, device="cuda")
            lse[rows] = ls.permute(2, 0, 1).reshape(n, self.Hq)
            # A score is a sum of D products that fp32 holds exactly (fp16: 22 bits, bf16: 16), added in fp32, truncated: D 2^-23 of what is
            # added; the exponent's product with scale and the difference to the maximum: 2 2^-23 of the largest score.  A weight is off
            # by that, by ex2's 2 ulp, and by its rounding to 16 bits (half a step; fp16 weights under 2^-14 by 2^-25 of the largest weight,
            # which the sum of weights is not below); the weighted sum and the sum of weights by an addition for each 8 tokens at most.
            T = k.shape[0]
            d = ((self.D + 4) * 2.0**-23 * size.masked_fill(~seen, 0.0).amax(-1)) if T else torch.zeros_like(ls)
            d = d.permute(2, 0, 1).reshape(n, self.Hq)
            chain = 2.0**-21 + (T / 8 + 16) * 2.0**-23
            bound[rows] = eps / 2 * o.abs() + ((eps / 2 + 2 * chain + 2 * d)[..., None] if T else 0.0) * a * (1 + eps)
            if self.q.dtype == torch.float16 and T:
                tiny = torch.einsum("nl,lhd->nhd", seen.double(), v.abs()) * 2.0**-25
                bound[rows] += tiny.repeat_interleave(R, 1) + 2.0**-25
            lbound[rows] = d + chain + 2.0**-22 * lse[rows].abs().nan_to_num(0.0, posinf=0.0)
        return out, lse, bound, lbound

    def check(self, scale=None, with_lse=True, **kw):
        scale = self.D ** -0.5 if scale is None else scale
        out = torch.full((self.n, self.Hq + 1, self.D), 7.0, dtype=self.q.dtype, device="cuda")[:, 1:]
        lse = torch.full((self.n, self.Hq), 7.0, dtype=torch.float32, device="cuda") if with_lse else None
        self.cache.attend(self.q, self.table, self.kv_len, cu_q=self.cu_q, prefix=self.prefix, scale=scale, out=out, lse=lse, **kw)
        assert self.cache.status() == dart.DART_OK
        want, wl, bound, lbound = self.reference(scale)
        mine = ~want.isnan()
        assert bool((out[~mine] == 7).all())
        off = (out.double() - want)[mine].abs()
        assert not off.isnan().any()
        assert bool((off <= bound[mine]).all()), "largest excess %.3g of %.3g" % (float((off - bound[mine]).max()), float(bound[mine].max()))
        if with_lse:
            none = wl == -math.inf
            assert bool((lse[none] == -math.inf).all()) and bool((lse[wl.isnan()] == 7).all())
            some = ~none & ~wl.isnan()
            assert bool(((lse.double() - wl)[some].abs() <= lbound[some]).all())
        return out, lse


DECODE = [
    # Hq, Hk, D, page, sequences
    (1, 1, 128, 16, [(1, 1)]), (8, 1, 128, 16, [(1, 5)]), (28, 4, 128, 16, [(1, 676)]), (32, 32, 128, 64, [(1, 33), (1, 1), (1, 400), (1, 31)]),
    (40, 40, 64, 32, [(1, 32), (1, 64), (1, 63), (1, 65), (1, 127), (1, 129)]), (16, 1, 128, 128, [(1, 1000), (1, 3)]), (17, 1, 64, 16, [(1, 250)]),
    (48, 2, 128, 256, [(1, 300), (1, 256), (1, 257)]), (12, 2, 64, 1024, [(1, 1023), (1, 1024), (1, 1025)]), (4, 4, 128, 16, [(1, n) for n in range(1, 70)]),
    (8, 8, 128, 16, [(1, 0), (1, 10), (1, 0)]), (2, 1, 128, 16, [(1, 20000)]), (32, 8, 128, 16, [(1, 517)] * 150),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", DECODE, ids=lambda c: "%dx%d_d%d_p%d_n%d" % (c[0], c[1], c[2], c[3], len(c[4])))
def test_single_tokens(dtype, case):
    Case(*case[:4], dtype, case[4]).check()


PROMPTS = [
    (4, 2, 128, 16, [(5, 5)]), (4, 4, 64, 16, [(1, 1), (2, 2), (17, 17), (64, 64)]), (7, 1, 128, 32, [(33, 50), (3, 200), (1, 7), (0, 9), (0, 0), (40, 40)]),
    (3, 3, 128, 16, [(6, 2), (4, 0), (9, 9)]), (8, 2, 128, 64, [(129, 129), (200, 300)]), (32, 8, 128, 16, [(77, 77), (21, 21), (50, 90)]), (2, 2, 64, 128, [(700, 700)]),
    (28, 4, 128, 16, [(257, 1000), (19, 19)]), (6, 1, 128, 256, [(300, 555)]), (1, 1, 128, 16, [(1000, 1000)]), (16, 4, 64, 16, [(130, 130)] * 5),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", PROMPTS, ids=lambda c: "%dx%d_d%d_p%d_n%d" % (c[0], c[1], c[2], c[3], len(c[4])))
def test_prompts_and_drafts(dtype, case):
    Case(*case[:4], dtype, case[4], gap=3).check()


SHARED = [
    # Hq, Hk, D, page, sequences, groups (sequences, prefix tokens), sequences before the first group
    (8, 2, 128, 16, [(1, 3), (1, 9)], [(2, 100)], 0), (28, 4, 128, 16, [(1, 5 + i) for i in range(48)], [(48, 1843)], 0),
    (4, 4, 64, 32, [(1, 1)] * 9, [(3, 31), (2, 32), (4, 33)], 0), (6, 2, 128, 16, [(1, 4)] * 7, [(2, 50), (0, 70), (3, 0), (1, 17)], 1),
    (32, 8, 128, 16, [(7, 7), (1, 12), (77, 77), (21, 30)], [(4, 298)], 0), (16, 1, 128, 64, [(5, 0), (1, 0), (3, 2)], [(3, 129)], 0),
    (8, 1, 64, 16, [(1, 40)] * 64, [(64, 5000)], 0), (5, 5, 128, 128, [(50, 50)] * 6, [(1, 300), (2, 10), (3, 1000)], 0), (2, 2, 128, 16, [(1, 1), (1, 0)], [(1, 1), (1, 0)], 0),
    (8, 2, 128, 16, [(300, 400), (2, 2)], [(2, 640)], 0), (40, 8, 128, 16, [(1, 77)] * 33, [(33, 777)], 0), (32, 32, 128, 16, [(3, 30)] * 20, [(10, 420), (10, 164)], 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", SHARED, ids=lambda c: "%dx%d_d%d_p%d_n%d_g%d" % (c[0], c[1], c[2], c[3], len(c[4]), len(c[5])))
def test_shared_prefixes(dtype, case):
    Case(*case[:4], dtype, case[4], groups=case[5], before=case[6], gap=1 if len(case[4]) > 3 else 0).check()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("sharp", [0.0, 8.0, 60.0])
@pytest.mark.parametrize("q", [1, 40])
def test_equal_and_peaked_scores(dtype, sharp, q):
    """All scores equal; a few tokens that take all the weight, so that the running maximum moves far."""
    Case(8, 2, 128, 16, dtype, [(q, 900), (q, 130), (q, q)], groups=[(2, 600), (1, 300)], sharp=sharp).check()
    Case(8, 2, 64, 16, dtype, [(q, 900), (q, 130), (q, q)], sharp=sharp).check()


def test_scales_and_strides():
    for scale in (1.0, 0.01, 1e-30):
        Case(4, 2, 128, 16, "bf16", [(3, 100), (1, 5)], groups=[(2, 70)], qstride=3, sharp=0.3).check(scale=scale)
    c = Case(4, 2, 64, 16, "fp16", [(1, 100), (1, 5)], qstride=2)
    wide = torch.full((2, c.table.shape[1] + 5), 2**30, dtype=torch.int32, device="cuda")
    wide[:, :c.table.shape[1]] = c.table
    c.table = wide[:, :c.table.shape[1]]
    c.check(with_lse=False)


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(seed):
    import random

    r = random.Random(seed)
    Hk = r.choice((1, 2, 3, 4, 8))
    R = r.choice((1, 1, 2, 3, 4, 7, 8, 16, 20))
    B = r.randint(1, 30)
    most = r.choice((1, 1, 8, 70, 300))
    seqs = []
    for _ in range(B):
        n = r.randint(0, most) if most > 1 else 1
        seqs.append((n, r.choice((n, n + r.randint(0, 300), max(0, n - r.randint(0, 3))))))
    if not sum(n for n, _ in seqs):
        seqs[0] = (1, 1)
    groups, left, before = [], B, 0
    if seed % 3:
        before = r.randint(0, min(2, B - 1))
        left -= before
        while left > 0 and len(groups) < 5:
            a = r.randint(0, left)
            groups.append((a, r.choice((0, r.randint(1, 50), r.randint(1, 900)))))
            left -= a
    c = Case(Hk * R, Hk, r.choice((64, 128)), r.choice((16, 32, 64, 128, 256)), r.choice(("bf16", "fp16")), seqs, groups=groups, before=before, seed=seed,
             gap=r.choice((0, 2)) if most > 1 else 0)
    a, la = c.check()
    b, lb = c.check()
    mine = slice(c.cu[0], c.cu[-1])
    assert torch.equal(a[mine], b[mine]) and torch.equal(la[mine], lb[mine])  # the same bits again


def test_offsets_beyond_32_bits():
    """A cache of 9 GB: byte offsets of its last pages need more than 33 bits."""
    n_pages, Hk, page, D = 9 << 14, 2, 128, 128
    k = torch.empty((n_pages, Hk, page, D), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    c = Case(4, Hk, D, page, "bf16", [(1, 300), (140, 300)], groups=[(2, 700)])
    keep = c.k, c.v
    top = n_pages - c.k.shape[0]
    for big, small in ((k, c.k), (v, c.v)):
        big[top:] = small
    c.k, c.v, c.cache = k, v, dart.PagedCache(k, v)
    for t in (c.table, c.ptable):
        t[t < 2**29] += top
    rows = torch.randn((3, Hk, D), device="cuda").to(torch.bfloat16)
    last = torch.full((3, 1), n_pages - 1, dtype=torch.int32, device="cuda")
    c.check()
    c.cache.append(rows, rows, last, start=torch.tensor([100, 101, 127], dtype=torch.int32, device="cuda"))
    assert c.cache.status() == dart.DART_OK
    assert torch.equal(k[-1][:, [100, 101, 127]], rows.transpose(0, 1)) and torch.equal(v[-1][:, [100, 101, 127]], rows.transpose(0, 1))
    del keep


def test_bad_pages_and_lengths_are_reported():
    c = Case(4, 2, 128, 16, "bf16", [(1, 100), (1, 40)], groups=[(2, 64)])
    want = c.check()[0].clone()
    good = c.table.clone()
    for bad in (-1, c.k.shape[0], 2**31 - 1):
        c.table[0, 3] = bad
        out = c.cache.attend(c.q, c.table, c.kv_len, prefix=c.prefix)
        assert c.cache.status() == dart.DART_ERR_CHECK
        assert bool(out.isfinite().all()) and torch.equal(out[1], want[1])
    c.table.copy_(good)
    for bad in (-5, 10**9):
        kv = c.kv_len.clone()
        kv[0] = bad
        narrow = torch.zeros((2, 7), dtype=torch.int32, device="cuda")
        narrow[:, :7] = torch.where(c.table[:, :7] < 2**29, c.table[:, :7], 0)
        c.k.nan_to_num_(0.0), c.v.nan_to_num_(0.0)
        out = c.cache.attend(c.q, narrow, kv, prefix=c.prefix)
        assert c.cache.status() == dart.DART_ERR_CHECK
        # (shared out among the workers in another way: two results, each off by half a step of the weights and of the output)
        off = (out[1].double() - want[1].double()).abs()
        assert bool(out.isfinite().all()) and bool((off <= 4 * 2.0**-8 * 4).all()) and float(c.v.abs().max()) < 8
    cu = torch.tensor([2, 0, 2], dtype=torch.int32, device="cuda")  # does not ascend: no fault, nothing out of bounds
    c.cache.attend(c.q, c.table, c.kv_len, cu_q=cu)
    c.cache.status()


def test_two_streams_and_two_graphs():
    cases = [Case(8, 2, 128, 16, "bf16", [(1, 200 + 31 * i)] * 8, groups=[(8, 500)], seed=i) for i in range(2)]
    cases += [Case(8, 2, 128, 16, "bf16", [(40, 200 + 31 * i)] * 8, groups=[(8, 500)], seed=i) for i in range(2)]
    call = lambda c, **kw: c.cache.attend(c.q, c.table, c.kv_len, cu_q=c.cu_q, prefix=c.prefix, **kw)  # noqa: E731
    want = [call(c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        got += [(i, call(c, stream=s)) for i, (c, s) in enumerate(zip(cases, streams))]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i, o in got)
    graphs, outs = [], []
    for c, s in zip(cases, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs.append(call(c))
        graphs.append(graph)
    for c in cases:
        c.q.neg_()
    torch.cuda.synchronize()
    want = [call(c) for c in cases]
    for _ in range(3):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    assert all(c.cache.status() == dart.DART_OK for c in cases)


def test_replays_follow_the_lengths():
    c = Case(8, 2, 64, 16, "fp16", [(1, 300), (1, 90)], groups=[(2, 200)])
    graph = torch.cuda.CUDAGraph()
    call = lambda: c.cache.attend(c.q, c.table, c.kv_len, prefix=c.prefix)  # noqa: E731
    call()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = call()
    for lens, shared in (((300, 1), 200), ((17, 90), 1), ((0, 33), 0), ((299, 88), 199)):
        c.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        c.prefix[1].fill_(shared)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, call())
        c.seqs, c.groups = [(1, n) for n in lens], [(2, shared)]
        c.check()


def test_wrong_arguments_are_refused():
    c = Case(4, 2, 128, 16, "bf16", [(1, 20), (1, 5)], groups=[(2, 30)])
    ok = dict(q=c.q, table=c.table, kv_len=c.kv_len, prefix=c.prefix)
    for bad in (dict(q=c.q.half()), dict(q=c.q[..., :64]), dict(q=c.q.cpu()), dict(table=c.table.long()), dict(kv_len=c.kv_len[:1]), dict(kv_len=c.kv_len.long()),
                dict(out=c.q[:1]), dict(lse=torch.zeros(2, 4, device="cuda").half()), dict(prefix=(c.ptable, c.prefix[1].long(), c.prefix[2])),
                dict(prefix=(c.ptable, c.prefix[1], c.prefix[2][:1])), dict(cu_q=torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            c.cache.attend(**{**ok, **bad})
    for bad in (dict(out=c.q), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(q=c.q[:1]), dict(q=c.q[:, :3]), dict(wait_limit=-1)):
        with pytest.raises(dart.DartError):
            c.cache.attend(**{**ok, **bad})
    none = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert c.cache.attend(c.q[:0], c.table, c.kv_len, cu_q=none).shape == (0, 4, 128)
    a = dart.dart_attend_args(n_rows=2)
    assert dart.dart_attend(c.cache._c, a, None, 0, ctypes.c_void_p(0)) == dart.DART_ERR_BAD_SHAPE


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("Hq,Hk,D,seqs,groups", [
    (20, 1, 128, [(1, 700), (1, 31)], []), (128, 1, 64, [(1, 300)], []), (130, 1, 64, [(1, 300)], []), (33, 1, 128, [(9, 200), (1, 3)], [(2, 260)]),
    (4, 4, 128, [(128, 128), (129, 129), (127, 300)], []), (4, 4, 64, [(255, 255), (256, 256), (257, 500)], []), (14, 2, 128, [(18, 18), (37, 64)], [(1, 127), (1, 129)]),
    (8, 8, 64, [(200, 200)] * 3, [(3, 1)]), (6, 3, 128, [(90, 0), (70, 35), (65, 64)], [(1, 0), (2, 250)]),
])
def test_wide_tiles_at_their_edges(dtype, Hq, Hk, D, seqs, groups):
    """Rows of one token that do and do not fill a tile of 128, more query heads a KV head than a tile has rows, sequences that end beside a tile's
    end, engines without rows or without a token to see."""
    Case(Hq, Hk, D, 16, dtype, seqs, groups=groups, gap=1).check()


@pytest.mark.parametrize("q,groups", [(1, True), (40, False), (140, False)])
def test_a_wait_that_runs_out_is_reported(q, groups):
    """A hand-over that is withheld on purpose (a barrier that one warp never arrives at): the kernel gives up after 20 ms, frees its tensor memory
    and says which wait it was; the next call is served."""
    c = Case(8, 2, 128, 16, "bf16", [(q, 400)] * (20 if groups else 2), groups=[(20, 900)] if groups else [])
    want = c.check()[0].clone()
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    p = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
    out = torch.zeros((c.n, 8, 128), dtype=torch.bfloat16, device="cuda")
    pt, pl, cg = c.prefix or (None, None, None)
    a = dart.dart_attend_args(p(c.q), p(out), None, c.q.stride(0), out.stride(0), c.n, 8, len(c.seqs), len(c.groups), p(c.cu_q), p(c.table), p(c.kv_len), p(cg), p(pt), p(pl),
                              c.table.stride(0), pt.stride(0) if groups else 0, 128 ** -0.5, 20000, p(status), 1)
    need = dart.dart_attend_workspace(c.cache._c, a)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    assert dart.dart_attend(c.cache._c, a, p(ws), need, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == dart.DART_OK
    torch.cuda.synchronize()
    got = status.tolist()
    assert got[0] == dart.DART_ERR_TIMEOUT and 110 <= got[1] <= 125, got
    again = c.check()[0]
    mine = slice(c.cu[0], c.cu[-1])
    assert torch.equal(again[mine], want[mine])


@pytest.mark.parametrize("q,groups", [(1, True), (40, False), (140, False)])
def test_a_kernel_that_gives_up_waits_for_its_queries(q, groups):
    """The products give up at the first tile whose queries they would wait for, so that the copy may still be under way when the others learn
    of it: the block has to wait for it before it ends.  The wait is named, and calls that follow at once, on the same SMs, are served."""
    c = Case(8, 2, 128, 16, "bf16", [(q, 400)] * (20 if groups else 2), groups=[(20, 900)] if groups else [])
    want = c.check()[0].clone()
    p = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
    out = torch.zeros((c.n, 8, 128), dtype=torch.bfloat16, device="cuda")
    pt, pl, cg = c.prefix or (None, None, None)
    status = torch.zeros((4, 4), dtype=torch.int32, device="cuda")
    again = []
    for one in status:
        a = dart.dart_attend_args(p(c.q), p(out), None, c.q.stride(0), out.stride(0), c.n, 8, len(c.seqs), len(c.groups), p(c.cu_q), p(c.table), p(c.kv_len), p(cg), p(pt),
                                  p(pl), c.table.stride(0), pt.stride(0) if groups else 0, 128 ** -0.5, 20000, p(one), 2)
        need = dart.dart_attend_workspace(c.cache._c, a)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        assert dart.dart_attend(c.cache._c, a, p(ws), need, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == dart.DART_OK
        again.append(c.cache.attend(c.q, c.table, c.kv_len, cu_q=c.cu_q, prefix=c.prefix))
    torch.cuda.synchronize()
    for got in status.tolist():
        assert got[0] == dart.DART_ERR_TIMEOUT and got[1] == 113, got  # kWaitQueries
    mine = slice(c.cu[0], c.cu[-1])
    assert all(torch.equal(x[mine], want[mine]) for x in again) and c.cache.status() == dart.DART_OK


def test_lines_of_more_than_2_30_tiles():
    """72 sequences of 2^29 tokens each, all of them in one page: 1.2e9 tiles of 32 tokens, of which every worker takes its share.  Queries of
    zeros: every token weighs the same, values of zeros: the answer is exact, the log-sum tells how many tokens were counted (a thread's
    sum of ones is exact below 2^24; four of them and the pieces of some 17 workers are added in fp32: 30 roundings of 2^-24, and those of the logarithm)."""
    n, page, pages = 72, 1024, 1 << 19
    k, v = torch.randn((2, 2, 1, page, 64), device="cuda").to(torch.bfloat16)
    v[0].zero_()
    cache = dart.PagedCache(k, v)
    table = torch.zeros((n, pages), dtype=torch.int32, device="cuda")
    kv_len = torch.tensor([pages * page - 37 * i for i in range(n)], dtype=torch.int32, device="cuda")
    out = torch.full((n, 1, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, 1), 7.0, device="cuda")
    cache.attend(torch.zeros_like(out), table, kv_len, out=out, lse=lse)
    assert cache.status() == dart.DART_OK
    assert bool((out == 0).all())
    assert bool(((lse[:, 0].double() - kv_len.double().log()).abs() <= 60 * 2.0**-24 + 21 * 2.0**-22).all())


POISONED = [
    # Hq, Hk, D, sequences, groups: whole and cut items of the narrow and the wide forms, and every way of joining
    (4, 2, 128, [(1, 1), (1, 2), (1, 0), (1, 40)], []), (4, 1, 64, [(1, 30000)], []), (16, 16, 64, [(1, 700 + i) for i in range(300)], []),
    (2, 1, 128, [(3, 2), (5, 9000)], []), (8, 8, 128, [(40, 400), (50, 20), (1, 1)], []), (8, 2, 64, [(120, 3000), (90, 60)], []), (4, 4, 128, [(700, 700), (300, 100)], []),
    (8, 2, 128, [(1, 3), (1, 0), (1, 70)], [(2, 100)]), (8, 8, 64, [(1, 30)] * 80, [(40, 300), (40, 0)]), (8, 2, 64, [(9, 9), (30, 31), (12, 4)] * 10, [(15, 800), (10, 0)]),
    (4, 4, 128, [(200, 300), (150, 0), (3, 1)], [(3, 900)]), (32, 32, 64, [(1, 5)] * 700, [(700, 50)]),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("value", [NAN, math.inf, -math.inf])
@pytest.mark.parametrize("case", POISONED, ids=lambda c: "%dx%d_d%d_n%d_g%d" % (c[0], c[1], c[2], len(c[3]), len(c[4])))
def test_queries_that_are_not_numbers(dtype, value, case):
    """A query that holds a NaN or an infinity has scores that are NaN or infinite (no key is zero there), and by the formula no softmax: its row
    is NaN, log-sum too, in every form and however its pieces are joined.  Rows that see nothing stay zeros; all others are as without it."""
    Hq, Hk, D, seqs, groups = case
    c = Case(Hq, Hk, D, 16, dtype, seqs, groups=groups)
    assert bool((c.k[:, :, :, 3] != 0).all())
    want, wl, bound, lbound = c.reference(D ** -0.5)
    bad = torch.zeros((c.n, Hq), dtype=torch.bool, device="cuda")
    for b, (n, _) in enumerate(seqs):
        for t in {0, n // 2, n - 1} - {-1}:
            if (b + t) % 5 != 4:
                bad[c.cu[b] + t, (b * 3 + t) % Hq] = True
    c.q[..., 3] = torch.where(bad, value, c.q[..., 3])
    lse = torch.full((c.n, Hq), 7.0, device="cuda")
    out = c.cache.attend(c.q, c.table, c.kv_len, cu_q=c.cu_q, prefix=c.prefix, lse=lse)
    assert c.cache.status() == dart.DART_OK
    none = wl == -math.inf
    assert bool((out[none] == 0).all()) and bool((lse[none] == -math.inf).all())
    lost = bad & ~none
    assert int(lost.sum()) > 0
    assert bool(out[lost].isnan().all()), "%d of %d rows" % (int((~out[lost].isnan()).any(-1).sum()), int(lost.sum()))
    assert bool(lse[lost].isnan().all())
    some = ~bad & ~none
    assert bool(((out.double() - want)[some].abs() <= bound[some]).all())
    assert bool(((lse.double() - wl)[some].abs() <= lbound[some]).all())


@pytest.mark.parametrize("before", [dart.DART_OK, dart.DART_ERR_CHECK])
@pytest.mark.parametrize("bad_page", [False, True])
@pytest.mark.parametrize("withhold", [1, 2])
def test_a_wait_that_runs_out_says_more_than_a_bad_page(withhold, bad_page, before):
    """TIMEOUT (rows are not valid) over CHECK (a page read as zeros), in whichever order they come."""
    c = Case(8, 2, 128, 16, "bf16", [(40, 400)] * 3)
    if bad_page:
        c.table[:, 7] = -1
    status = torch.tensor([before, 0, 0, 0], dtype=torch.int32, device="cuda")
    p = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
    out = torch.zeros((c.n, 8, 128), dtype=torch.bfloat16, device="cuda")
    a = dart.dart_attend_args(p(c.q), p(out), None, c.q.stride(0), out.stride(0), c.n, 8, 3, 0, p(c.cu_q), p(c.table), p(c.kv_len), None, None, None, c.table.stride(0), 0,
                              128 ** -0.5, 20000, p(status), withhold)
    need = dart.dart_attend_workspace(c.cache._c, a)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    assert dart.dart_attend(c.cache._c, a, p(ws), need, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == dart.DART_OK
    torch.cuda.synchronize()
    got = status.tolist()
    assert got[0] == dart.DART_ERR_TIMEOUT and 110 <= got[1] <= 125, got


def test_what_a_call_reports_does_not_hide_a_wait_that_ran_out():
    """A cache's status word is shared by its calls: rows left out, pages that read as zeros, lengths that are cut and offsets that cannot be come
    after a TIMEOUT that nobody has read."""
    c = Case(4, 2, 128, 16, "bf16", [(1, 100), (1, 40)])
    wide = Case(4, 2, 128, 16, "bf16", [(40, 100), (40, 40)])
    rows = torch.zeros((2, 2, 128), dtype=torch.bfloat16, device="cuda")
    bad = torch.full_like(c.table, -1)
    long = torch.full_like(c.kv_len, 1 << 20)
    none = torch.zeros_like(c.table)
    calls = [
        lambda: c.cache.append(rows, rows, bad), lambda: c.cache.attend(c.q, bad, c.kv_len), lambda: c.cache.attend(c.q, none, long), lambda: c.cache.attend(c.q, none, -long),
        lambda: c.cache.attend(wide.q, torch.full_like(wide.table, -1)[:, :c.table.shape[1]].contiguous(), wide.kv_len, cu_q=wide.cu_q),
    ]
    for call in calls:
        call()
        assert c.cache.status() == dart.DART_ERR_CHECK  # (each of them does report)
        c.cache._status[0] = dart.DART_ERR_TIMEOUT
        call()
        assert c.cache.status() == dart.DART_ERR_TIMEOUT and c.cache.status() == dart.DART_OK


def test_tables_that_are_the_last_columns_of_wider_ones():
    """The table of a view whose last row ends beyond its memory is copied on the call's stream; a length that is longer than its row is cut there."""
    c = Case(4, 2, 64, 16, "fp16", [(1, 100), (1, 40)], groups=[(2, 70)])
    want = c.check()[0].clone()
    views = []
    for t in (c.table, c.ptable):
        wide = torch.full((t.shape[0], t.shape[1] + 5), 2**30, dtype=torch.int32, device="cuda")
        wide[:, 5:] = t
        views.append(wide[:, 5:])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (None, s):
        torch.cuda._sleep(10_000_000)
        out = c.cache.attend(c.q, views[0], c.kv_len, prefix=(views[1], *c.prefix[1:]), stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and c.cache.status() == dart.DART_OK
    c.k.nan_to_num_(0.0), c.v.nan_to_num_(0.0)
    views[0][views[0] >= c.k.shape[0]] = 0
    out = c.cache.attend(c.q, views[0], torch.full_like(c.kv_len, 16 * views[0].shape[1] + 1), prefix=(views[1], *c.prefix[1:]))
    cut = c.cache.attend(c.q, views[0].contiguous(), torch.full_like(c.kv_len, 16 * views[0].shape[1]), prefix=c.prefix)
    assert c.cache.status() == dart.DART_ERR_CHECK and torch.equal(out, cut)


@pytest.mark.parametrize("q", [1, 30])
@pytest.mark.parametrize("which,offsets", [
    ("q", [0, 2, 1, 4]), ("q", [0, 3, 3, 5]), ("q", [-1, 1, 2, 4]), ("q", [0, 0, 5, 4]), ("q", [4, 0, 4, 0]), ("q", [0, 2**31 - 1, 2, 4]),
    ("group", [0, 2, 1, 3]), ("group", [0, 1, 2, 4]), ("group", [-1, 1, 2, 3]), ("group", [3, 0, 0, 3]), ("group", [1, 1, 1, 0]),
])
@pytest.mark.parametrize("prefixes", [False, True])
def test_offsets_that_cannot_be_are_reported(which, offsets, prefixes, q):
    """Offsets that descend, or leave the rows or sequences that there are: reported, and not a row is written, in no form and by no join."""
    if which == "group" and not prefixes:
        pytest.skip("no groups")
    c = Case(8, 2, 64, 16, "bf16", [(q, 90), (2 * q, 200), (q, 50)], groups=[(1, 300), (1, 40), (1, 0)] if prefixes else [])
    bad = torch.tensor([x * q if abs(x) < 2**30 else x for x in offsets] if which == "q" else offsets, dtype=torch.int32, device="cuda")
    cu = bad if which == "q" else c.cu_q
    prefix = (*c.prefix[:2], bad) if which == "group" else c.prefix
    out, lse = torch.full_like(c.q, 7.0), torch.full((c.n, 8), 7.0, device="cuda")
    c.cache.attend(c.q, c.table, c.kv_len, cu_q=cu, prefix=prefix, out=out, lse=lse)
    assert c.cache.status() == dart.DART_ERR_CHECK
    assert bool((out == 7).all()) and bool((lse == 7).all())
    c.check()


def test_threads_call_at_once():
    import threading

    cases = [Case(8, 2, 128, 16, "bf16", [(n, 300 + 17 * i)] * 6, groups=[(6, 500)], seed=i) for i, n in enumerate((1, 40, 1, 40))]
    want = [c.check(with_lse=False)[0].clone() for c in cases]
    bad = []

    def work(c, w):
        s = torch.cuda.Stream()
        for _ in range(20):
            out = c.cache.attend(c.q, c.table, c.kv_len, cu_q=c.cu_q, prefix=c.prefix, stream=s)
            s.synchronize()
            if not torch.equal(out, w):
                bad.append(c)

    threads = [threading.Thread(target=work, args=x) for x in zip(cases, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_from_projection_to_answer():
    """The operators as they are used together: keys normalised and rotated, scored and reduced; the kept rows into pages; questions about each image
    behind its shared, shortened prompt; then a decoding step."""
    B, S, Hq, Hk, D, P, Kp, vo, nv, Q = 2, 260, 8, 2, 64, 4, 50, 12, 220, 3
    g = _gen(77)
    rows = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    inv = (1.0 / 10000.0 ** (torch.arange(0, D, 2, dtype=torch.float64) / D)).float().cuda()
    rope, w = dart.Rope(inv), (1 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16)
    k0, v0, hidden = rows(B * S, Hk, D), rows(B * S, Hk, D), rows(B, S, Hk * D)
    pos = torch.arange(S, device="cuda").repeat(B)
    _, keys = dart.norm_rope(None, k0, pos=pos, rope=rope, k_weight=w)
    ctx = dart.Dart(B, S, Hk * D, P, Kp)
    out_hidden, idx, out_pos = ctx.reduce(hidden, keys.view(B, S, Hk * D), vo, nv, P, Kp)
    S_out = S - nv + Kp
    n_seq, per = B * Q, (S_out + 15) // 16
    kc, vc = rows(B * per + n_seq * 2, Hk, 16, D), rows(B * per + n_seq * 2, Hk, 16, D)
    ids = torch.randperm(kc.shape[0], generator=g, device="cuda").to(torch.int32)
    ptable, table = ids[:B * per].view(B, per), ids[B * per:].view(n_seq, 2)
    cache = dart.PagedCache(kc, vc)
    cache.append(k0, v0, ptable, idx=idx, S=S, pos=out_pos, rope=rope, k_weight=w)  # from the rows before the rotation: the same keys
    prefix = (ptable, torch.full((B,), S_out, dtype=torch.int32, device="cuda"), torch.arange(0, n_seq + 1, Q, dtype=torch.int32, device="cuda"))
    have, own_k, own_v = 0, [[] for _ in range(n_seq)], [[] for _ in range(n_seq)]
    for n in (13, 1, 1):  # the questions, then two tokens of the answers
        q1, k1, v1 = rows(n_seq * n, Hq, D), rows(n_seq * n, Hk, D), rows(n_seq * n, Hk, D)
        at = (S + have + torch.arange(n, device="cuda")).repeat(n_seq)
        q2, k2 = dart.norm_rope(q1, k1, pos=at, rope=rope, q_weight=w, k_weight=w)
        start = torch.full((n_seq,), have, dtype=torch.int32, device="cuda")
        cache.append(k1, v1, table, start=start, pos=at, rope=rope, k_weight=w)
        have += n
        cu = torch.arange(0, n_seq * n + 1, n, dtype=torch.int32, device="cuda")
        out = cache.attend(q2, table, start + n, cu_q=cu, prefix=prefix)
        assert cache.status() == dart.DART_OK and ctx.status() == dart.DART_OK
        for s in range(n_seq):
            own_k[s].append(k2[s * n:(s + 1) * n]), own_v[s].append(v1[s * n:(s + 1) * n])
            b = s // Q
            kept = idx[b].long()
            K = torch.cat([keys.view(B, S, Hk, D)[b, kept]] + own_k[s]).double().repeat_interleave(Hq // Hk, 1)
            V = torch.cat([v0.view(B, S, Hk, D)[b, kept]] + own_v[s]).double().repeat_interleave(Hq // Hk, 1)
            x = q2[s * n:(s + 1) * n].double()
            logits = torch.einsum("nhd,lhd->hnl", x, K) / D ** 0.5
            hidden_from = S_out + have - n + torch.arange(n, device="cuda") + 1
            logits = logits.masked_fill(torch.arange(K.shape[0], device="cuda")[None, :] >= hidden_from[:, None], -math.inf)
            p = logits.softmax(-1)
            want, size = torch.einsum("hnl,lhd->nhd", p, V), torch.einsum("hnl,lhd->nhd", p, V.abs())
            # output and weights rounded to bf16: half a step each; the scores' sums of 64 products in fp32: 68 * 2^-23 of |q||k| / 8 <= 20
            bound = 2.0**-8 * want.abs() + (2.0**-8 + 2 * 68 * 2.0**-23 * 20 + 1e-4) * size * (1 + 2.0**-8)
            off = (out[s * n:(s + 1) * n].double() - want).abs()
            assert bool((off <= bound).all()) and float(x.norm(dim=-1).max() * K.norm(dim=-1).max()) / 8 < 20
    assert torch.equal(out_hidden, torch.gather(hidden, 1, idx.long()[..., None].expand(-1, -1, Hk * D)))
    ctx.close()


def test_keys_of_grouped_heads_are_reduced_by_themselves():
    """Fewer key heads than query heads: keys narrower than the hidden rows.  The reduction takes the keys as its rows, its index list then packs the
    hidden rows and names the rows that go into pages."""
    B, S, Hq, Hk, D, P, Kp, vo, nv = 3, 240, 8, 2, 64, 4, 40, 20, 200
    g = _gen(5)
    rows = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    rope = dart.Rope((1.0 / 10000.0 ** (torch.arange(0, D, 2, dtype=torch.float64) / D)).float().cuda())
    hidden, k, v = rows(B, S, Hq * D), rows(B * S, Hk, D), rows(B * S, Hk, D)
    pos = torch.arange(S, device="cuda").repeat(B)
    _, keys = dart.norm_rope(None, k, pos=pos, rope=rope)
    ctx = dart.Dart(B, S, Hk * D, P, Kp)
    kept_keys, idx, out_pos = ctx.reduce(keys.view(B, S, Hk * D), None, vo, nv, P, Kp)
    S_out = S - nv + Kp
    out_hidden = torch.empty((B, S_out, Hq * D), dtype=torch.bfloat16, device="cuda")
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert dart.dart_gather_rows(hidden.data_ptr(), ctypes.cast(idx.data_ptr(), ctypes.POINTER(ctypes.c_int32)), B, S, S_out, 2 * Hq * D, out_hidden.data_ptr(), 0,
                                 stream) == dart.DART_OK
    per = (S_out + 15) // 16
    kc, vc = rows(B * per, Hk, 16, D), rows(B * per, Hk, 16, D)
    table = torch.randperm(B * per, generator=g, device="cuda").to(torch.int32).view(B, per)
    cache = dart.PagedCache(kc, vc)
    cache.append(k, v, table, idx=idx, S=S, pos=out_pos, rope=rope)
    assert cache.status() == dart.DART_OK and ctx.status() == dart.DART_OK
    assert torch.equal(out_hidden, torch.gather(hidden, 1, idx.long()[..., None].expand(-1, -1, Hq * D)))
    t = torch.arange(S_out, device="cuda")
    for b in range(B):
        page = table[b].long()[t // 16]
        assert torch.equal(kc[page, :, t % 16].reshape(S_out, -1), kept_keys[b])  # the same rows, rotated on the way
        assert torch.equal(vc[page, :, t % 16], v.view(B, S, Hk, D)[b, idx[b].long()])
    ctx.close()
