"""The paged KV cache on the GPU, through the C ABI, against plain 64-bit forms (tests/paged_oracle.py, which also derives the
tolerances).  Every cache is NaN where no query may look."""
import math

import pytest
import torch

import paged_oracle as oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def spa():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_21233_amd as m
    m.load_library()
    return m


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------- block tables and slot maps
def _plan_both(spa, table, ctx, new, free, free_range, n_tokens, page, n_pages):
    want = oracle.plan(table, ctx, new, free, free_range, n_tokens, page, n_pages)
    mine = table.cuda()
    got = spa.paged_plan(mine, _i32(ctx), _i32(new), _i32(free), _i32(free_range), n_tokens, page, n_pages)
    for name, g, w in zip(("table", "q_starts", "kv_lens", "slots", "positions", "taken"), (mine, *got), want):
        assert torch.equal(g.cpu(), w), name


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("batch,longest,more", [(1, 0, 1), (1, 1000, 1), (3, 100, 300), (63, 500, 1), (64, 70, 40), (65, 3, 17), (257, 900, 30), (4096, 40, 3)])
def test_plan_takes_pages_in_order(spa, page, batch, longest, more):
    g = torch.Generator().manual_seed(batch + page)
    draw = lambda hi: torch.randint(0, hi + 1, (batch,), generator=g).tolist()  # noqa: E731
    ctx, new = draw(longest), draw(more)
    C = (longest + more) // page + 2
    n_pages = batch * C + 5
    ids = torch.randperm(n_pages, generator=g)
    table = ids[:batch * C].view(batch, C).to(torch.int32)
    free = torch.randperm(n_pages, generator=g).tolist()
    n_tokens = sum(new) + 9                                       # the last nine are padding
    _plan_both(spa, table, ctx, new, free, [2, len(free)], n_tokens, page, n_pages)
    for room in (0, 1, (sum(new) // page + 1) // 2):               # too few pages for some
        _plan_both(spa, table, ctx, new, free, [3, 3 + room], n_tokens, page, n_pages)


@pytest.mark.parametrize("ctx,new,n_tokens", [
    ([0, 10, 5], [0, 0, 0], 1),                                   # nothing new
    ([-1, 10, 5], [3, 4, 5], 12), ([7, 10, 5], [3, -4, 5], 12),    # negative lengths
    ([7, 10, 5], [3, 4, 5], 6), ([7, 10, 5], [3, 2 ** 31 - 1, 5], 20),      # more tokens than the packed rows hold
    ([2 ** 31 - 1, 60, 5], [3, 4, 5], 12), ([7, 10, 5], [3, 400, 5], 500),  # past the table
    ([64, 63, 1], [64, 1, 127], 192),                              # ends on a page's border
])
def test_plan_leaves_out_what_does_not_fit(spa, ctx, new, n_tokens):
    table = torch.arange(6, dtype=torch.int32).view(3, 2)
    _plan_both(spa, table, ctx, new, [9, 8, 7, 6, 5], [0, 5], n_tokens, 64, 10)


def test_plan_of_wild_tables_and_ranges(spa):
    table = torch.tensor([[-3, 50, 0], [2 ** 31 - 1, 1, 2]], dtype=torch.int32)
    for free_range in ([0, 2], [-5, 90], [1, 0], [7, 9], [2, 2]):
        _plan_both(spa, table, [100, 20], [30, 60], [-1, 12, 3], free_range, 95, 64, 10)
    mine = table.cuda()                                            # no free list at all
    got = spa.paged_plan(mine, _i32([100, 20]), _i32([20, 40]), _i32([]), _i32([0, 0]), 60, 64, 10)
    want = oracle.plan(table, [100, 20], [20, 40], [], [0, 0], 60, 64, 10)
    assert torch.equal(mine.cpu(), want[0]) and all(torch.equal(g.cpu(), w) for g, w in zip(got, want[1:]))


def test_plan_of_a_table_with_wider_rows(spa):
    wide = torch.full((5, 12), -9, dtype=torch.int32, device="cuda")
    ctx, new = [10, 0, 200, 64, 3], [100, 5, 7, 1, 130]
    table = wide[:, 2:8]
    want = oracle.plan(table.cpu(), ctx, new, list(range(20)), [0, 20], 300, 64, 20)
    spa.paged_plan(table, _i32(ctx), _i32(new), _i32(list(range(20))), _i32([0, 20]), 300, 64, 20)
    assert torch.equal(wide[:, 2:8].cpu(), want[0])
    assert (wide[:, :2] == -9).all() and (wide[:, 8:] == -9).all()


# --------------------------------------------------------------------------------------------------------------- append
def _bits(*shape, seed=0):
    """bf16 values of any bits, NaN payloads among them"""
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-2 ** 15, 2 ** 15, shape, generator=g).to(torch.int16).view(torch.bfloat16)


def _same_bits(a, b):
    return torch.equal(a.cpu().view(torch.int16), b.cpu().view(torch.int16))


def _slot_maps(n_pages, page):
    g = torch.Generator().manual_seed(n_pages * page)
    n = n_pages * page
    any_order = torch.randperm(n, generator=g)
    yield any_order[:n // 2].tolist()                              # scattered
    yield list(range(5, n - 6))                                    # one run that starts and ends inside a piece
    yield [s if s % 5 else -1 for s in range(3, n // 2)]           # padding in between
    yield [n, -1, 2 ** 31 - 1, -2 ** 31, 7]                        # outside the cache
    yield [n - 1]
    yield list(range(7, -1, -1)) + list(range(n - 20, n - 12))     # a run backwards, an aligned one later


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("page,heads,n_pages", [(16, 1, 20), (32, 3, 9), (64, 8, 5), (128, 2, 7)])
def test_append_moves_the_bits(spa, head_dim, page, heads, n_pages):
    for turn, slots in enumerate(_slot_maps(n_pages, page)):
        T = len(slots)
        k, v = _bits(T, heads, head_dim, seed=turn), _bits(T, heads, head_dim, seed=50 + turn)
        k_pages, vt_pages = _bits(n_pages, heads, page, head_dim, seed=90), _bits(n_pages, heads, head_dim, page, seed=91)
        want = oracle.append(k, v, torch.tensor(slots), k_pages, vt_pages)
        mine = k_pages.cuda(), vt_pages.cuda()
        spa.paged_append(k.cuda(), v.cuda(), _i32(slots), *mine)
        assert _same_bits(mine[0], want[0]) and _same_bits(mine[1], want[1]), turn


def test_append_of_strided_tensors(spa):
    """K and V out of one projection's output, or of a prefill's [batch, heads, tokens, dim]; pages of both in one allocation."""
    T, H, D, page, N = 150, 4, 128, 64, 6
    qkv = _bits(T, 3 * H, D + 16, seed=1).cuda()
    k, v = qkv[:, H:2 * H, :D], _bits(1, H, T, D, seed=2).cuda()[0].transpose(0, 1)
    both = _bits(N, 2, H, page * D, seed=3).cuda()
    before = both.clone()
    k_pages, vt_pages = both[:, 0].view(N, H, page, D), both[:, 1].view(N, H, D, page)
    slots = [17 + t for t in range(T)]
    want = oracle.append(k.cpu(), v.cpu(), torch.tensor(slots), k_pages.cpu(), vt_pages.cpu())
    spa.paged_append(k, v, _i32(slots), k_pages, vt_pages)
    assert _same_bits(k_pages, want[0]) and _same_bits(vt_pages, want[1])
    assert not _same_bits(both, before)


# ------------------------------------------------------------------------------------------------------------ attention
def _attn_close(spa, step, lse=True, new=None, **how):
    call = dict(softmax_scale=how.get("scale"), n_sink_tokens=how.get("sink", 0), window_tokens=how.get("window", 0),
                softcap=how.get("softcap", 0.0), slopes=None if how.get("slopes") is None else how["slopes"].cuda())
    out = torch.full((step.T, *step.q.shape[1:]), 7.0, dtype=torch.bfloat16, device="cuda")
    got = spa.paged_attn(step.q.cuda(), step.k_pages.cuda(), step.vt_pages.cuda(), step.table.cuda(), _i32(step.starts), _i32(step.kv_lens),
                         max_new_tokens=new or 0, return_lse=lse, out=out, **call)
    want, want_lse, tol, lse_tol = step.want(**how)
    end = step.starts[-1]
    assert (out[end:] == 7.0).all(), "padding"
    off = (out.cpu().double() - want)[:end].abs() - tol[:end]
    assert not torch.isnan(off).any() and off.max().item() <= 0, (off.max().item(), (off == off.max()).nonzero()[0].tolist())
    if lse:
        g, w = got[1].cpu().double()[:end], want_lse[:end]
        assert torch.equal(torch.isinf(g), torch.isinf(w))
        off = torch.where(torch.isinf(w), 0.0, (g - w).abs() - lse_tol[:end])
        assert off.max().item() <= 0, (off.max().item(), (off == off.max()).nonzero()[0].tolist())
    return out


DECODE = [[0], [1], [14, 15, 16], [63, 64, 65, 0, 31, 32], [500], [127, 128, 255, 256, 1000, 3, 2047, 2500]]


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("ctx", DECODE, ids=lambda c: "-".join(map(str, c))[:20])
def test_attn_of_single_tokens(spa, ctx, page, head_dim):
    step = oracle.Step(sum(ctx) + page, ctx, [1] * len(ctx), page=page, head_dim=head_dim, padding=2, peak=3.0)
    _attn_close(spa, step, new=1)


@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (8, 8), (5, 1), (10, 2), (16, 1), (17, 1), (32, 1), (33, 1), (40, 1), (70, 1), (96, 3)])
def test_attn_of_head_layouts(spa, q_heads, kv_heads):
    step = oracle.Step(q_heads, [300, 77, 0], [1, 1, 1], q_heads=q_heads, kv_heads=kv_heads, head_dim=64)
    _attn_close(spa, step, new=1)
    step = oracle.Step(q_heads, [300, 77, 0], [3, 40, 9], q_heads=q_heads, kv_heads=kv_heads, head_dim=64)
    _attn_close(spa, step, new=40)


CHUNKS = [([0], [2]), ([5], [16]), ([64], [64]), ([100], [33]), ([0], [300]), ([1000], [129]), ([31, 700, 0], [5, 64, 130]),
          ([900, 20, 64, 0, 333], [1, 200, 1, 1, 7]), ([10, 0, 50], [0, 12, 0])]


@pytest.mark.parametrize("head_dim,page,q_heads,kv_heads", [(128, 64, 4, 2), (64, 16, 6, 2), (128, 32, 5, 1), (64, 128, 2, 2), (128, 16, 8, 1), (64, 64, 4, 1)])
@pytest.mark.parametrize("ctx,new", CHUNKS, ids=lambda c: "-".join(map(str, c)))
def test_attn_of_chunks(spa, ctx, new, head_dim, page, q_heads, kv_heads):
    step = oracle.Step(sum(ctx) + sum(new), ctx, new, page=page, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, padding=3)
    a = _attn_close(spa, step, new=max(new))
    b = _attn_close(spa, step, new=0)                  # whatever the host knows of the lengths
    c = _attn_close(spa, step, new=1, lse=False)
    end = step.starts[-1]
    assert torch.isfinite(a[:end]).all() and torch.isfinite(b[:end]).all() and torch.isfinite(c[:end]).all()


@pytest.mark.parametrize("sink,window", [(0, 1), (0, 17), (4, 1), (64, 64), (70, 100), (1, 128), (200, 33), (5000, 7), (0, 5000), (2 ** 31 - 1, 2 ** 31 - 1), (0, 2 ** 31 - 1), (128, 300)])
@pytest.mark.parametrize("ctx,new", [([700], [1]), ([0, 63, 64, 1500, 400], [1, 1, 1, 1, 1]), ([650], [150]), ([900, 20, 300], [1, 90, 33])], ids=lambda c: "-".join(map(str, c)))
def test_attn_sees_sinks_and_window_only(spa, ctx, new, sink, window):
    for page, head_dim in ((16, 64), (64, 128)):
        step = oracle.Step(sink % 1000 + window % 1000, ctx, new, page=page, head_dim=head_dim, q_heads=4, kv_heads=1)
        step.hide(sink, window, new)
        _attn_close(spa, step, new=max(new), sink=sink, window=window)


@pytest.mark.parametrize("softcap,slopes,window", [(20.0, False, 0), (0.5, False, 0), (0.0, True, 0), (30.0, True, 0), (5.0, True, 90), (1e-3, False, 0), (1e4, False, 10)])
@pytest.mark.parametrize("ctx,new", [([700, 3], [1, 1]), ([130, 0, 600], [140, 33, 1])], ids=lambda c: "-".join(map(str, c)))
def test_attn_with_capped_logits_and_bias_by_distance(spa, ctx, new, softcap, slopes, window):
    step = oracle.Step(int(softcap), ctx, new, q_heads=8, kv_heads=2, page=32, peak=6.0)
    s = torch.exp2(-torch.arange(1.0, 9.0)) if slopes else None
    _attn_close(spa, step, new=max(new), softcap=softcap, slopes=s, window=window, sink=3)


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("softcap,slopes", [(0.0, False), (0.0, True), (25.0, False), (25.0, True)])
def test_attn_of_every_kernel(spa, softcap, slopes, page, head_dim):
    """Requests of few and of many rows in one call, only few, only many; with and without cuts."""
    s = torch.exp2(-torch.arange(1.0, 5.0)) if slopes else None
    for ctx, new in (([130, 0, 700], [140, 33, 1]), ([200, 33, 900], [1, 1, 2]), ([650], [90])):
        step = oracle.Step(page + len(ctx), ctx, new, q_heads=4, kv_heads=1, page=page, head_dim=head_dim, peak=2.0)
        _attn_close(spa, step, new=max(new), softcap=softcap, slopes=s)


@pytest.mark.parametrize("softcap", [1e-38, 1e-44, 65536.0])
def test_attn_of_the_smallest_and_largest_cap(spa, softcap):
    step = oracle.Step(1, [100, 0], [1, 40], q_heads=4, kv_heads=1, head_dim=64)
    step.q[0] = 0.0
    _attn_close(spa, step, new=40, softcap=softcap)


def test_attn_with_wild_slopes(spa):
    """Slopes that favour far keys, none, large ones."""
    step = oracle.Step(5, [400, 90], [1, 70], q_heads=4, kv_heads=1, head_dim=64)
    _attn_close(spa, step, new=70, slopes=torch.tensor([-0.25, 0.0, 40.0, 1e-6]))


@pytest.mark.parametrize("new", [[1, 1], [5, 150]], ids=["1", "150"])
@pytest.mark.parametrize("scale", [0.5, 3.0, 1e-4])
def test_attn_of_peaked_and_flat_rows(spa, new, scale):
    """Logits of some hundreds: the reference of the running softmax moves."""
    step = oracle.Step(int(scale * 10), [600, 200], new, q_heads=4, kv_heads=1, peak=8.0)
    _attn_close(spa, step, new=max(new), scale=scale)


@pytest.mark.parametrize("new", [1, 150])
def test_attn_of_logits_that_grow_along_the_keys(spa, new):
    step = oracle.Step(9, [1500], [new], q_heads=2, kv_heads=1, head_dim=64)
    n = step.kv_lens[0]
    step.q = (torch.full_like(step.q, 0.25) + step.q / 16).to(torch.bfloat16)
    ramp = (torch.arange(n)[None, :, None] * (600.0 / n)).to(torch.bfloat16)      # logits up to 0.25 * 64 * 600 / 8 = 1200
    for sign in (1, -1):
        step.keys = [(step.keys[0] / 8 + sign * ramp).to(torch.bfloat16)]
        for j in range(-(-n // 64)):
            at = slice(64 * j, min(64 * j + 64, n))
            step.k_pages[step.table[0, j], :, :at.stop - at.start] = step.keys[0][:, at]
        _attn_close(spa, step, new=new)


def test_attn_of_rows_that_see_nothing(spa):
    """Requests without a key, and more new tokens than cached ones: zeros and -inf, no NaN."""
    for new in ([1, 1, 1], [40, 200, 7]):
        step = oracle.Step(2, [0, 70, 33], new, q_heads=4, kv_heads=2, page=16, head_dim=64)
        step.kv_lens = [0, new[1] - 1, 0 if new[2] == 1 else 3]
        _attn_close(spa, step, new=max(new))


@pytest.mark.parametrize("long", [1, 40])
def test_attn_over_a_long_cache_is_cut_and_merged(spa, long):
    step = oracle.Step(long, [20000, 30, 5000, 0], [long, 1, 1, 2], q_heads=4, kv_heads=1, head_dim=64, page=128)
    _attn_close(spa, step, new=long)
    _attn_close(spa, step, new=long, window=9000, sink=300)


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("q_heads", [4, 16, 20, 32, 40])
def test_attn_of_one_long_request_is_cut_and_merged(spa, q_heads, head_dim):
    """One KV head: few workgroups, that make a part of the dims each, of 16, 32 or more rows."""
    for ctx in (3000, 600, 511):
        step = oracle.Step(q_heads, [ctx], [1], q_heads=q_heads, kv_heads=1, head_dim=head_dim, page=32)
        _attn_close(spa, step, new=1)
        _attn_close(spa, step, new=1, softcap=20.0, window=700, sink=70)


def test_attn_of_two_thousand_requests(spa):
    g = torch.Generator().manual_seed(4)
    ctx, new = torch.randint(0, 40, (2000,), generator=g).tolist(), torch.randint(0, 3, (2000,), generator=g).tolist()
    ctx[1500], new[1500], new[700] = 3000, 1, 60
    step = oracle.Step(2000, ctx, new, q_heads=2, kv_heads=1, head_dim=64, page=16)
    _attn_close(spa, step, new=60)


def test_attn_of_many_requests(spa):
    g = torch.Generator().manual_seed(1)
    ctx = torch.randint(0, 200, (300,), generator=g).tolist()
    ctx[17] = 6000
    new = [1 + (b % 50 == 7) * 30 for b in range(300)]
    step = oracle.Step(300, ctx, new, q_heads=2, kv_heads=1, head_dim=64, page=32)
    _attn_close(spa, step, new=31)


def test_attn_of_strided_tensors(spa):
    step = oracle.Step(3, [200, 90], [1, 20], q_heads=6, kv_heads=2, page=64)
    T, N = step.T, step.k_pages.shape[0]
    qkv = torch.full((T, 10, 144), math.nan, dtype=torch.bfloat16, device="cuda")
    qkv[:, 2:8, 8:136] = step.q.cuda()
    both = torch.empty((N, 2, 2, 64 * 128), dtype=torch.bfloat16, device="cuda")
    both[:, 0], both[:, 1] = step.k_pages.cuda().flatten(2), step.vt_pages.cuda().flatten(2)
    wide = torch.full((2, 50), -1, dtype=torch.int32, device="cuda")
    wide[:, 3:3 + step.table.shape[1]] = step.table.cuda()
    room = torch.full((6, T, 160), 7.0, dtype=torch.bfloat16, device="cuda")
    out = room[:, :, 16:144].transpose(0, 1)
    got = spa.paged_attn(qkv[:, 2:8, 8:136], both[:, 0].view(N, 2, 64, 128), both[:, 1].view(N, 2, 128, 64), wide[:, 3:3 + step.table.shape[1]],
                         _i32(step.starts), _i32(step.kv_lens), out=out)
    plain = spa.paged_attn(step.q.cuda(), step.k_pages.cuda(), step.vt_pages.cuda(), step.table.cuda(), _i32(step.starts), _i32(step.kv_lens))
    assert torch.equal(got.view(torch.int16), plain.view(torch.int16))
    assert (room[:, :, :16] == 7.0).all() and (room[:, :, 144:] == 7.0).all()


def test_attn_of_infinite_and_nan_values(spa):
    """A single query meets what it sees, and nothing else; a NaN key or query makes its rows NaN, no other ones."""
    step = oracle.Step(4, [100, 100, 300], [1, 1, 1], q_heads=2, kv_heads=1, head_dim=64)
    clean = spa.paged_attn(step.q.cuda(), step.k_pages.cuda(), step.vt_pages.cuda(), step.table.cuda(), _i32(step.starts), _i32(step.kv_lens))
    step.vt_pages[step.table[0, 0], 0, 5, 3] = math.inf
    step.k_pages[step.table[1, 1], 0, 2, 9] = math.nan
    got = spa.paged_attn(step.q.cuda(), step.k_pages.cuda(), step.vt_pages.cuda(), step.table.cuda(), _i32(step.starts), _i32(step.kv_lens))
    assert torch.equal(got[2], clean[2]) and torch.isnan(got[1]).all()
    assert torch.isinf(got[0, :, 5]).all() and torch.equal(got[0, :, :5], clean[0, :, :5]) and torch.equal(got[0, :, 6:], clean[0, :, 6:])


@pytest.mark.parametrize("head_dim,page,q_heads", [(64, 16, 4), (128, 64, 4), (128, 32, 2), (64, 128, 24)])
@pytest.mark.parametrize("ctx,new,window,sink", [(100, 4, 0, 0), (300, 7, 40, 3), (5, 150, 0, 0), (70, 150, 33, 70), (700, 130, 300, 10), (2000, 40, 0, 0)])
def test_values_that_are_not_finite_reach_those_who_see_them_and_no_others(spa, ctx, new, window, sink, head_dim, page, q_heads):
    step = oracle.Step(new, [ctx], [new], page=page, q_heads=q_heads, kv_heads=1, head_dim=head_dim)
    call = lambda: spa.paged_attn(step.q.cuda(), step.k_pages.cuda(), step.vt_pages.cuda(), step.table.cuda(), _i32(step.starts), _i32(step.kv_lens),  # noqa: E731
                                  max_new_tokens=new, window_tokens=window, n_sink_tokens=sink).float().cpu()
    clean, n = call(), ctx + new
    odd = {n - 1: (3, math.inf), n - new // 2: (9, math.nan), n - new + 1: (60, -math.inf), max(0, n - new - window - 1): (17, math.inf), 1: (33, -math.inf),
           n - 3: (3, -math.inf)}
    for key, (d, value) in odd.items():
        step.vt_pages[step.table[0, key // page], 0, d, key % page] = value
    got = call()
    for i in range(new):
        pos, want = ctx + i, clean[i].clone()
        seen = {key for key in odd if key <= pos and (window == 0 or pos - key < window or key < sink)}
        for d in {odd[key][0] for key in seen}:
            mixed = sum(odd[key][1] for key in seen if odd[key][0] == d)
            if math.isnan(mixed):
                assert torch.isnan(got[i, :, d]).all()
            else:                                                  # a weight of 0 makes NaN of an infinite value
                assert (torch.isnan(got[i, :, d]) | (got[i, :, d] == mixed)).all(), (i, d)
            want[:, d] = got[i, :, d]
        assert torch.equal(want.nan_to_num(7.0), got[i].nan_to_num(7.0)), i


def test_attn_of_malformed_lengths_stays_inside(spa):
    """Unspecified rows, but every other request keeps its bits."""
    step = oracle.Step(6, [100, 50, 80], [1, 1, 1], q_heads=4, kv_heads=1, head_dim=64)
    t = (step.q.cuda(), step.k_pages.cuda(), step.vt_pages.cuda())
    clean = spa.paged_attn(*t, step.table.cuda(), _i32(step.starts), _i32(step.kv_lens))
    table = step.table.clone()
    table[1] = torch.tensor([2 ** 31 - 1, -2 ** 31])
    for kv in ([101, 10 ** 9, 81], [101, -5, 81], [101, 2 ** 31 - 1, 81]):
        got = spa.paged_attn(*t, table.cuda(), _i32(step.starts), _i32(kv))
        assert torch.equal(got[0], clean[0]) and torch.equal(got[2], clean[2])
    for starts in ([0, 1, 2, 10 ** 9], [-5, 1, 2, 3], [0, 3, 1, 3], [2, 1, 0, 0], [0, 2 ** 31 - 1, -2 ** 31, 3]):
        spa.paged_attn(*t, step.table.cuda(), _i32(starts), _i32(step.kv_lens), max_new_tokens=1)
        spa.paged_attn(*t, step.table.cuda(), _i32(starts), _i32(step.kv_lens))
    torch.cuda.synchronize()


def test_attn_far_past_32_bit_offsets(spa):
    """Pages behind the first 4 GiB of the cache."""
    page, H, D = 128, 1, 128
    n_pages = 5 * 2 ** 30 // (page * H * D * 2)
    step = oracle.Step(8, [700], [1], page=page, q_heads=2, kv_heads=H, head_dim=D)
    k = torch.zeros((n_pages, H, page, D), dtype=torch.bfloat16, device="cuda")
    vt = torch.zeros((n_pages, H, D, page), dtype=torch.bfloat16, device="cuda")
    table = step.table.clone()
    for j in range(table.shape[1]):
        there = n_pages - 1 - 3 * j
        k[there], vt[there] = step.k_pages[table[0, j]].cuda(), step.vt_pages[table[0, j]].cuda()
        table[0, j] = there
    near = spa.paged_attn(step.q.cuda(), step.k_pages.cuda(), step.vt_pages.cuda(), step.table.cuda(), _i32(step.starts), _i32(step.kv_lens))
    far = spa.paged_attn(step.q.cuda(), k, vt, table.cuda(), _i32(step.starts), _i32(step.kv_lens))
    assert torch.equal(near, far)
    x = _bits(3, H, D, seed=5)
    slots = [n_pages * page - 1, (n_pages - 2) * page + 7, 2 ** 24 + 5]
    spa.paged_append(x.cuda(), x.cuda(), _i32(slots), k, vt)
    for t, s in enumerate(slots):
        assert _same_bits(k[s // page, :, s % page], x[t]) and _same_bits(vt[s // page, :, :, s % page], x[t])


# -------------------------------------------------------------------------------------- as they are used, one after the other
def test_a_prefill_and_the_steps_after_it(spa):
    """Prompts through the prefill with every block selected, their K and V into pages, then chunks and single tokens: every
    step's output is what dense attention of the whole sequence has at its positions."""
    g = torch.Generator().manual_seed(12)
    page, Hq, Hkv, D, lens = 64, 8, 2, 128, [500, 130]
    total = [n + 200 for n in lens]
    randn = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16)  # noqa: E731
    q, k, v = ([randn(h, n, D) for n in total] for h in (Hq, Hkv, Hkv))
    C = -(-max(total) // page)
    n_pages = 2 * C + 1
    table = torch.full((2, C), -1, dtype=torch.int32, device="cuda")
    k_pages = torch.full((n_pages, Hkv, page, D), math.nan, dtype=torch.bfloat16, device="cuda")
    vt_pages = torch.full((n_pages, Hkv, D, page), math.nan, dtype=torch.bfloat16, device="cuda")
    free = torch.randperm(n_pages, generator=g).to(torch.int32).cuda()
    used, have = 0, [0, 0]
    outs = [[], []]
    for new in (lens, [100, 1], [1, 64], [1, 1], [33, 90], [1, 1]):
        rows = [[x[b][:, have[b]:have[b] + new[b]] for b in range(2)] for x in (q, k, v)]
        qs, ks, vs = (torch.cat([r.transpose(0, 1) for r in x]).cuda() for x in rows)
        starts, kv_lens, slots, positions, taken = spa.paged_plan(table, _i32(have), _i32(new), free, _i32([used, n_pages]), sum(new), page, n_pages)
        spa.paged_append(ks, vs, slots, k_pages, vt_pages)
        out = spa.paged_attn(qs, k_pages, vt_pages, table, starts, kv_lens, max_new_tokens=max(new))
        assert positions.tolist() == [have[b] + i for b in range(2) for i in range(new[b])]
        for b in range(2):
            outs[b].append(out[starts[b]:starts[b + 1]].cpu())
            have[b] += new[b]
        used += int(taken[0])
        assert int(taken[1]) == 0 and kv_lens.tolist() == have
    for b in range(2):
        n = have[b]
        want, _, tol, _ = oracle.attn(q[b][:, :n].transpose(0, 1), [k[b][:, :n]], [v[b][:, :n]], [0, n], [n])
        off = (torch.cat(outs[b]).double() - want).abs() - tol
        assert off.max().item() <= 0
        prefill = spa.fused(q[b][None, :, :lens[b]].cuda(), k[b][None, :, :lens[b]].cuda(), v[b][None, :, :lens[b]].cuda(), 64, 1, 1, 4096)[0]
        first = outs[b][0].transpose(0, 1).double()
        # the prefill rounds weights and output as this kernel does: each is within the tolerance of the exact value
        assert ((prefill.cpu().double() - first).abs() - 2 * tol[:lens[b]].transpose(0, 1)).max().item() <= 0


def test_a_captured_step_replays_with_other_lengths(spa):
    """Plan, append and attention in one graph, with one workspace; eager work of the same kind in between."""
    page, Hq, Hkv, D, B, C = 16, 8, 2, 64, 5, 40
    n_pages = B * C
    g = torch.Generator().manual_seed(3)
    table = torch.randperm(n_pages, generator=g).view(B, C).to(torch.int32).cuda()
    k_pages = torch.randn((n_pages, Hkv, page, D), generator=g).to(torch.bfloat16).cuda()
    vt_pages = torch.randn((n_pages, Hkv, D, page), generator=g).to(torch.bfloat16).cuda()
    ctx, new = _i32([0] * B), _i32([1] * B)
    free, free_range, T = _i32(list(range(n_pages))), _i32([0, 0]), 40
    q, k, v = (torch.randn((T, h, D), generator=g).to(torch.bfloat16).cuda() for h in (Hq, Hkv, Hkv))

    def step():
        starts, kv_lens, slots, *_ = spa.paged_plan(table, ctx, new, free, free_range, T, page, n_pages)
        spa.paged_append(k, v, slots, k_pages, vt_pages)
        return spa.paged_attn(q, k_pages, vt_pages, table, starts, kv_lens, return_lse=True) + (starts,)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for turn, (c, n) in enumerate([([15, 0, 300, 64, 9], [1, 1, 1, 1, 1]), ([600, 20, 0, 0, 630], [1, 30, 0, 7, 2]), ([1, 2, 3, 4, 5], [0, 0, 0, 0, 0]),
                                   ([600, 20, 500, 400, 639], [1, 9, 12, 3, 1])]):
        # pages that the requests have cover the new tokens, so the free list stays out of it: ctx is rounded up to its page below
        c = [min(x, C * page - y) for x, y in zip(c, n)]
        c = [x if (x + y + page - 1) // page == (x + page - 1) // page else (x + y + page - 1) // page * page - y for x, y in zip(c, n)]
        ctx.copy_(_i32(c))
        new.copy_(_i32(n))
        free_range.copy_(_i32([0, n_pages]))
        q.copy_(torch.randn(q.shape, generator=g).to(torch.bfloat16))
        graph.replay()
        again = step()
        torch.cuda.synchronize()
        end = int(again[2][-1])
        assert torch.equal(got[2], again[2])
        assert torch.equal(got[0][:end].view(torch.int16), again[0][:end].view(torch.int16)) and torch.equal(got[1][:end], again[1][:end]), turn


def test_calls_on_two_streams_do_not_meet(spa):
    step = oracle.Step(11, [3000, 200], [1, 60], q_heads=8, kv_heads=2, head_dim=64)
    t = [x.cuda() for x in (step.q, step.k_pages, step.vt_pages, step.table)] + [_i32(step.starts), _i32(step.kv_lens)]
    want = spa.paged_attn(*t)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for turn in range(6):
        with torch.cuda.stream(streams[turn % 2]):
            got.append(spa.paged_attn(*t))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got)


def test_results_repeat_bit_for_bit(spa):
    step = oracle.Step(13, [9000, 200, 0], [1, 90, 3], q_heads=8, kv_heads=2)
    t = [x.cuda() for x in (step.q, step.k_pages, step.vt_pages, step.table)] + [_i32(step.starts), _i32(step.kv_lens)]
    a, b = (spa.paged_attn(*t, return_lse=True) for _ in range(2))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
