"""Norm and rotation of queries and keys, and rows on their way into a paged cache, against the formulas in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2502_11494_b200 import dart  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _inv_freq(rot, base=10000.0):
    return (1.0 / base ** (torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()


def reference(x, w, eps, pos, inv_freq, sections, interleaved):
    """(z, size): the rotated rows in fp64 and, per element, the size of what its sum adds up."""
    y = x.double()
    if w is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w.double()
    size = y.abs().clone()
    if inv_freq is None:
        return y, size
    half = inv_freq.numel()
    pos = pos.reshape(-1, x.shape[0])
    axis = torch.cat([torch.full((n,), a) for a, n in enumerate(sections or (half,))]).to(x.device)
    angle = (pos.double()[axis] * inv_freq.double()[:, None]).T[:, None, :]
    i = torch.arange(half, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    z = y.clone()
    z[..., a] = y[..., a] * angle.cos() - y[..., b] * angle.sin()
    z[..., b] = y[..., b] * angle.cos() + y[..., a] * angle.sin()
    size[..., a] = size[..., b] = y[..., a].abs() + y[..., b].abs()
    return z, size


def close(got, want, size):
    """One rounding to the type (half a step), and fp32 on the way: the sum of squares, root, quotient, two products and a
    sum are within 16 roundings of 2^-24 (a head's sum of at most 256 squares is taken in threads of 16 and a tree: 20 more on a
    square, 10 on its root), the angle's rounding to fp32 (at most half a turn, 2^-24 of it: 2 pi 2^-25 = 1.9e-7) and sincospif's 2
    roundings: 30 * 2^-24 + 2e-7 = 2e-6 of what is added up."""
    step = torch.finfo(got.dtype).eps / 2
    tiny = torch.finfo(got.dtype).smallest_normal * step  # half a step among the subnormal numbers
    bound = (step * want.abs() + 2e-6 * size) * (1 + step) + tiny
    off = (got.double() - want).abs()
    assert not off.isnan().any()
    assert bool((off <= bound).all()), "largest excess %.3g" % float((off - bound).max())


def _rows(shape, dtype, g):
    return (torch.randn(shape, generator=g, device="cuda") * 2).to(dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n,Hq,Hk,D,rot,interleaved,norm", [
    (1, 1, 1, 128, 128, False, True), (1, 28, 4, 128, 128, False, True), (16, 32, 32, 128, 128, False, False),
    (7, 5, 3, 64, 64, True, True), (33, 3, 1, 64, 32, False, True), (5, 40, 40, 128, 64, True, True), (3, 2, 1, 80, 80, False, True),
    (9, 7, 0, 96, 96, True, False), (9, 0, 7, 96, 48, False, True), (2, 1, 1, 256, 256, False, True), (11, 4, 2, 256, 16, True, True),
    (4, 3, 2, 8, 0, False, True), (4, 3, 2, 24, 16, False, True), (4, 3, 2, 72, 64, False, True), (4, 65, 2, 16, 16, True, False),
    (677, 12, 2, 128, 128, False, True), (4099, 3, 1, 128, 128, True, True), (1201, 32, 8, 64, 64, False, True), (2, 2, 1, 128, 0, False, False),
])
def test_norm_and_rotation(dtype, n, Hq, Hk, D, rot, interleaved, norm):
    g = _gen(n * 31 + D)
    dt = TYPES[dtype]
    qkv = _rows((n, Hq + Hk + 2, D), dt, g)  # columns of a wider buffer
    q, k = (qkv[:, :Hq] if Hq else None), (qkv[:, Hq:Hq + Hk] if Hk else None)
    w = [(1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(dt) if norm else None for _ in range(2)]
    pos = torch.randint(-5, 100000, (n,), generator=g, device="cuda")
    inv = _inv_freq(rot) if rot else None
    rope = dart.Rope(inv, interleaved=interleaved) if rot else None
    before = qkv.clone()
    out = dart.norm_rope(q, k, pos=pos if rot else None, rope=rope, q_weight=w[0] if Hq else None, k_weight=w[1] if Hk else None, eps=1e-5)
    torch.cuda.synchronize()
    assert torch.equal(qkv.view(torch.int16), before.view(torch.int16))
    for x, o, wx in ((q, out[0], w[0]), (k, out[1], w[1])):
        if x is None:
            assert o is None
            continue
        close(o, *reference(x, wx, 1e-5, pos, inv, None, interleaved))


@pytest.mark.parametrize("sections", [(16, 24, 24), (0, 64, 0), (64, 0, 0), (1, 2, 61), (40, 24)])
def test_positions_on_several_axes(sections):
    g = _gen(5)
    n, D = 130, 128
    q, k = _rows((n, 4, D), torch.bfloat16, g), _rows((n, 2, D), torch.bfloat16, g)
    wide = torch.randint(0, 5000, (len(sections), n + 9), generator=g, device="cuda")
    pos = wide[:, :n]  # axes further apart than rows
    inv = _inv_freq(D)
    got = dart.norm_rope(q, k, pos=pos, rope=dart.Rope(inv, sections=sections))
    for x, o in zip((q, k), got):
        close(o, *reference(x, None, 0, pos, inv, sections, False))


def test_far_positions_turn_exactly():
    """Positions beyond what fp32 counts: the angle is a product in fp64 (2^-53 of 2^40 radians is 1e-4; 2^33 leaves 1e-6)."""
    g = _gen(6)
    pos = torch.tensor([0, 1, 2**24 + 1, 2**31 + 7, -(2**31) - 9, 2**33 + 1], device="cuda")
    q = _rows((6, 2, 64), torch.float16, g)
    inv = _inv_freq(64)
    got, _ = dart.norm_rope(q, None, pos=pos, rope=dart.Rope(inv))
    want, size = reference(q, None, 0, pos, inv, None, False)
    close(got, want, 2 * size)  # (2^33 radians are themselves held to 2^-53: 1e-6 of what is added up, on top)


def test_in_place_and_into_columns():
    g = _gen(7)
    qkv = _rows((50, 12, 128), torch.bfloat16, g)
    pos = torch.arange(50, device="cuda")
    rope = dart.Rope(_inv_freq(128))
    w = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    want = dart.norm_rope(qkv[:, :8], qkv[:, 8:10], pos=pos, rope=rope, q_weight=w)
    cols = torch.full_like(qkv, 7.0)
    dart.norm_rope(qkv[:, :8], qkv[:, 8:10], pos=pos, rope=rope, q_weight=w, out=(cols[:, 1:9], cols[:, 10:12]))
    v = qkv[:, 10:].clone()
    dart.norm_rope(qkv[:, :8], qkv[:, 8:10], pos=pos, rope=rope, q_weight=w, out=(qkv[:, :8], qkv[:, 8:10]))
    assert torch.equal(cols[:, 1:9], want[0]) and torch.equal(cols[:, 10:12], want[1]) and bool((cols[:, 0] == 7).all() and (cols[:, 9] == 7).all())
    assert torch.equal(qkv[:, :8], want[0]) and torch.equal(qkv[:, 8:10], want[1]) and torch.equal(qkv[:, 10:], v)


def test_zero_rows_and_rows_of_zeros():
    q = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    got, none = dart.norm_rope(q, None, q_weight=w, eps=1e-6)
    assert none is None and bool((got == 0).all())
    assert dart.norm_rope(q[:0], None, q_weight=w)[0].shape == (0, 2, 64)


def test_wrong_tensors_are_refused():
    q = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    rope = dart.Rope(_inv_freq(64))
    pos = torch.arange(3, device="cuda")
    for bad in (dict(q=q.float()), dict(q=q.transpose(0, 1)), dict(q=q[..., ::2]), dict(pos=pos[:2]), dict(pos=pos.int()), dict(pos=None),
                dict(q_weight=torch.ones(32, dtype=torch.bfloat16, device="cuda")), dict(q_weight=torch.ones(64, device="cuda")),
                dict(q=q.cpu()), dict(q=None), dict(out=(q[:, :1], None))):
        a = dict(q=q, k=None, pos=pos, rope=rope)
        a.update(bad)
        with pytest.raises(ValueError):
            dart.norm_rope(**a)
    with pytest.raises(dart.DartError):
        dart.norm_rope(q, None, out=(q.view(-1)[:2 * 64].view(1, 2, 64).expand(3, 2, 64), None))


# ---- the paged cache -----------------------------------------------------------------------------------------------------------

def _cache(n_pages, Hk, page, D, dt, g):
    return _rows((n_pages, Hk, page, D), dt, g), _rows((n_pages, Hk, page, D), dt, g)


def _tables(lengths, page, g, spare=3):
    need = [(n + page - 1) // page for n in lengths]
    width = max(1, max(need)) + 2
    total = sum(need) + spare
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lengths), width), 2**30, dtype=torch.int32, device="cuda")  # entries that nobody may read
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, total


def _append_reference(kc, vc, k, v, rows, table, page, start, idx, S, pos, w, inv, cu0=0):
    K, V = kc.double(), vc.double()
    size = torch.zeros_like(K)
    touched = torch.zeros(K.shape[:1] + K.shape[2:3], dtype=torch.bool, device=K.device)
    n = cu0
    for b, r in enumerate(rows):
        for t in range(r):
            slot = start[b] + t
            src = b * S + int(idx[n]) if idx is not None else n
            p = torch.tensor([slot if pos is None else int(pos[n])], device=K.device)
            pg, at = int(table[b, slot // page]), slot % page
            z, s = reference(k[src][None], w, 1e-6, p, inv, None, False)
            K[pg, :, at], size[pg, :, at] = z[0], s[0]
            V[pg, :, at] = v[src].double()
            touched[pg, at] = True
            n += 1
    return K, V, size, touched


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,start,Hk,D,page,S,rot,norm", [
    ([1], [0], 1, 128, 16, 0, 128, False), ([1] * 5, [0, 15, 16, 17, 700], 4, 128, 16, 0, 128, True), ([3, 0, 1, 40, 0], [2, 9, 0, 31, 0], 2, 64, 32, 0, 64, True),
    ([0, 0], [1, 0], 2, 64, 16, 0, 0, False), ([20, 20], [0, 0], 8, 128, 64, 50, 128, False), ([13, 1, 29], [5, 0, 16], 3, 80, 7, 31, 80, True),
    ([65], [255], 2, 256, 256, 0, 32, False), ([9, 9, 9], [0, 1, 2], 40, 128, 1, 9, 0, False), ([300, 7], [1, 2], 5, 24, 128, 0, 16, True),
])
def test_rows_go_to_their_slots(dtype, rows, start, Hk, D, page, S, rot, norm):
    g = _gen(sum(rows) + D)
    dt = TYPES[dtype]
    table, total = _tables([a + b for a, b in zip(rows, start)], page, g)
    kc, vc = _cache(total, Hk, page, D, dt, g)
    n = sum(rows)
    src = len(rows) * S if S else n
    kv = _rows((src, 2 * Hk, D), dt, g)
    idx = pos = None
    if S:
        idx = torch.cat([torch.randperm(S, generator=g, device="cuda")[:r].sort().values for r in rows]).to(torch.int32)
        pos = idx.long() * 3 + 1
    equal = len(set(rows)) == 1 and rows[0] > 0
    cu = None if equal else torch.tensor([sum(rows[:b]) for b in range(len(rows) + 1)], dtype=torch.int32, device="cuda")
    w = (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(dt) if norm else None
    inv = _inv_freq(rot) if rot else None
    K, V, size, touched = _append_reference(kc, vc, kv[:, :Hk], kv[:, Hk:], rows, table, page, start, idx, S, pos, w, inv)
    old = kc.clone()
    cache = dart.PagedCache(kc, vc)
    cache.append(kv[:, :Hk], kv[:, Hk:], table, start=torch.tensor(start, dtype=torch.int32, device="cuda") if any(start) else None, cu_rows=cu, idx=idx, S=S,
                 pos=pos, rope=dart.Rope(inv) if rot else None, k_weight=w, eps=1e-6)
    assert cache.status() == dart.DART_OK
    assert torch.equal(vc.double(), V)
    t = touched[:, None, :, None].expand_as(kc)
    assert torch.equal(kc[~t], old[~t])
    if n:
        close(kc[t], K[t], size[t])


def test_rows_behind_the_last_sequence_are_left_alone():
    g = _gen(9)
    table, total = _tables([8, 8], 16, g)
    kc, vc = _cache(total, 2, 16, 64, torch.bfloat16, g)
    k = _rows((30, 2, 64), torch.bfloat16, g)
    cu = torch.tensor([4, 9, 12], dtype=torch.int32, device="cuda")  # rows 0..3 and 12..29 belong to nobody
    K, V, _, _ = _append_reference(kc, vc, k, k, [5, 3], table, 16, [0, 0], None, 0, None, None, None, cu0=4)
    cache = dart.PagedCache(kc, vc)
    cache.append(k, k, table, cu_rows=cu)
    assert cache.status() == dart.DART_OK
    assert torch.equal(kc.double(), K) and torch.equal(vc.double(), V)


def test_bad_pages_and_rows_are_left_out_and_reported():
    g = _gen(10)
    kc, vc = _cache(4, 1, 16, 64, torch.bfloat16, g)
    old = kc.clone()
    cache = dart.PagedCache(kc, vc)
    k = _rows((4, 1, 64), torch.bfloat16, g)
    good = torch.tensor([[0], [1], [2], [3]], dtype=torch.int32, device="cuda")
    for table, start, idx in ((torch.tensor([[0], [4], [-1], [2**31 - 1]], dtype=torch.int32, device="cuda"), None, None),
                              (good, torch.tensor([0, 16, -1, 2**31 - 1], dtype=torch.int32, device="cuda"), None),
                              (good, None, torch.tensor([0, 1, -1, 2**31 - 1], dtype=torch.int32, device="cuda"))):
        kc.copy_(old)
        cache.append(k, k, table, start=start, idx=idx, S=1 if idx is not None else 0)
        assert cache.status() == dart.DART_ERR_CHECK and cache.status() == dart.DART_OK
        want = old.clone()
        want[0, 0, 0] = k[0, 0]
        assert torch.equal(kc, want)


def test_kept_rows_of_a_reduction_go_into_pages():
    """A reduction's own outputs as they are: out_idx, out_pos and, with independent pivots, cu_seqlens; and the other stream."""
    B, S, H, D, P, Kp, vo, nv = 3, 180, 4, 64, 4, 40, 10, 150
    g = _gen(11)
    q, keys = _rows((B * S, H, D), torch.bfloat16, g), _rows((B * S, H, D), torch.bfloat16, g)
    v = _rows((B * S, H, D), torch.bfloat16, g)
    inv = _inv_freq(D)
    pos = torch.arange(S, device="cuda").repeat(B)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        _, turned = dart.norm_rope(q, keys, pos=pos, rope=dart.Rope(inv))
        ctx = dart.Dart(B, S, H * D, P, Kp)
        cu = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
        rows = turned.view(B, S, H * D)
        for opts in (None, dart.dart_opts(rule=dart.DART_RULE_UNION, cu_seqlens=cu.data_ptr())):
            _, idx, out_pos = ctx.reduce(rows, rows, vo, nv, P, Kp, opts=opts)
            S_out = S - nv + Kp
            table = torch.arange(B * 5, dtype=torch.int32, device="cuda").view(B, 5)
            kc, vc = _cache(B * 5, H, 16, D, torch.bfloat16, g)
            cache = dart.PagedCache(kc, vc)
            cache.append(turned, v, table, cu_rows=cu if opts else None, idx=idx, S=S, pos=out_pos)
            assert cache.status() == dart.DART_OK and ctx.status() == dart.DART_OK
            lens = (cu[1:] - cu[:-1]).tolist() if opts else [S_out] * B
            first = 0
            for b in range(B):
                kept = idx.flatten()[first:first + lens[b]].long() if opts else idx[b].long()
                first += lens[b]
                got = kc[table[b].long()].permute(0, 2, 1, 3).reshape(-1, H, D)[:lens[b]]
                assert torch.equal(got, turned.view(B, S, H, D)[b, kept])
                got = vc[table[b].long()].permute(0, 2, 1, 3).reshape(-1, H, D)[:lens[b]]
                assert torch.equal(got, v.view(B, S, H, D)[b, kept])
        ctx.close()


def test_captured_and_replayed():
    g = _gen(12)
    k = _rows((4, 2, 128), torch.bfloat16, g)
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(4, 2)
    kc, vc = _cache(8, 2, 16, 128, torch.bfloat16, g)
    start = torch.zeros(4, dtype=torch.int32, device="cuda")
    cache, rope = dart.PagedCache(kc, vc), dart.Rope(_inv_freq(128))
    out = torch.empty_like(k)
    pos = torch.arange(4, device="cuda")
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        cache.append(k, k, table, start=start, rope=rope)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            dart.norm_rope(None, k, pos=pos, rope=rope, out=(None, out))
            cache.append(out, k, table, start=start)
    for step in (3, 17, 31):
        start.fill_(step)
        k.copy_(_rows((4, 2, 128), torch.bfloat16, g))
        graph.replay()
        torch.cuda.synchronize()
        _, want = dart.norm_rope(None, k, pos=pos, rope=rope)
        for b in range(4):
            assert torch.equal(kc[table[b, step // 16], :, step % 16], want[b]) and torch.equal(vc[table[b, step // 16], :, step % 16], k[b])
    assert cache.status() == dart.DART_OK and math.isfinite(float(out.float().sum()))


def _busy_block(nbytes):
    """A block of the current stream's that is free again, but whose last user is still to come: behind some 50 ms of nothing."""
    t = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    t.fill_(7)
    return t.data_ptr()


def test_outputs_are_made_on_the_stream_that_writes_them():
    """With stream= and no out=: memory that the current stream has freed but not finished with is not handed to another stream."""
    n, Hq, Hk, D = 4096, 8, 2, 128
    g = _gen(3)
    q, k = torch.randn((n, Hq, D), generator=g, device="cuda").to(torch.bfloat16), torch.randn((n, Hk, D), generator=g, device="cuda").to(torch.bfloat16)
    rope, pos = dart.Rope(_inv_freq(D)), torch.arange(n, device="cuda")
    want = dart.norm_rope(q, k, pos=pos, rope=rope)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        blocks = {_busy_block(q.numel() * 2), _busy_block(k.numel() * 2)}
        got = dart.norm_rope(q, k, pos=pos, rope=rope, stream=s)
        s.synchronize()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and not {t.data_ptr() for t in got} & blocks
        del got
    q_only, none = dart.norm_rope(q, None, pos=pos, rope=rope, stream=s)
    s.synchronize()
    assert none is None and torch.equal(q_only, want[0])


def test_positions_are_copied_on_the_stream_that_reads_them():
    """Positions [B, S_out] that lie apart are copied for the call, on the call's stream: a copy queued behind the current stream's work would be
    read before it is made."""
    B, S_out, Hk, D, page = 2, 300, 2, 64, 16
    g = _gen(4)
    k, v = _rows((B * S_out, Hk, D), torch.bfloat16, g), _rows((B * S_out, Hk, D), torch.bfloat16, g)
    pages = B * ((S_out + page - 1) // page)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(B, -1)
    wide = torch.randint(0, 5000, (B, S_out + 7), generator=g, device="cuda")
    rope, s = dart.Rope(_inv_freq(D)), torch.cuda.Stream()
    results = []
    for stream in (None, s):
        kc = torch.zeros((pages, Hk, page, D), dtype=torch.bfloat16, device="cuda")
        cache = dart.PagedCache(kc, torch.zeros_like(kc))
        torch.cuda.synchronize()
        if stream is not None:
            torch.cuda._sleep(100_000_000)  # some 50 ms
        cache.append(k, v, table, pos=wide[:, :S_out], rope=rope, stream=stream)
        torch.cuda.synchronize()
        assert cache.status() == dart.DART_OK
        results.append(kc)
    assert torch.equal(*results)


def _bad_append(cache, **kw):
    rows = torch.zeros((2, cache.heads, cache.head_dim), dtype=cache.dtype, device="cuda")
    cache.append(rows, rows, torch.full((2, 1), -1, dtype=torch.int32, device="cuda"), **kw)


def test_reports_of_other_threads_are_not_lost():
    """Another thread's call comes between the reading of the status and its clearing: what it reports is read the next time."""
    import threading

    k = torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16, device="cuda")
    cache = dart.PagedCache(k, torch.zeros_like(k))

    class Word:
        """The status word; before it is cleared the other thread gets half a second to report."""

        def __init__(self, t):
            self.t, self.thread = t, None

        def __getitem__(self, i):
            return self.t[i]

        def zero_(self):
            self.thread = threading.Thread(target=lambda: (_bad_append(cache), torch.cuda.synchronize()))
            self.thread.start()
            self.thread.join(0.5)
            return self.t.zero_()

    word = cache._status = Word(cache._status)
    _bad_append(cache)
    assert cache.status() == dart.DART_ERR_CHECK
    word.thread.join()
    cache._status = word.t
    assert cache.status() == dart.DART_ERR_CHECK and cache.status() == dart.DART_OK


def test_a_new_cache_can_be_used_on_another_stream_at_once():
    """The status word is cleared before the first call may report, whatever the stream that was current has still to do."""
    k = torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16, device="cuda")
    v, s = torch.zeros_like(k), torch.cuda.Stream()
    with torch.cuda.stream(s):
        _bad_append(dart.PagedCache(k, v))  # (memory of the stream's own is there: asking the device for some would wait)
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)  # some 50 ms
    cache = dart.PagedCache(k, v)
    with torch.cuda.stream(s):
        _bad_append(cache)
    s.synchronize()
    assert cache.status() == dart.DART_ERR_CHECK and cache.status() == dart.DART_OK


def test_as_many_rows_as_there_are_numbers():
    """2^31 - 1 rows of one head of 8, in place: 34 GB, rows counted up to the largest number that n_rows can be."""
    n = 2**31 - 1
    rows = torch.zeros((n, 1, 8), dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, 7, 8, 2**30 + 5, n - 9, n - 8, n - 7, n - 2, n - 1], device="cuda")
    x = _rows((len(at), 1, 8), torch.bfloat16, _gen(9))
    rows[at] = x
    w = torch.arange(1, 9, device="cuda").to(torch.bfloat16)
    q, none = dart.norm_rope(rows, None, q_weight=w, eps=1e-6, out=(rows, None))
    torch.cuda.synchronize()
    assert q is rows and none is None
    close(rows[at], *reference(x, w, 1e-6, None, None, None, False))
    assert bool((rows[2:7] == 0).all()) and bool((rows[n - 6:n - 2] == 0).all())
