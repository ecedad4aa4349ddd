"""The quantised paged cache and shared prompts on the GPU, through the C ABI, against plain 64-bit forms (tests/paged_q8_oracle.py;
tests/paged_oracle.py derives the attention's tolerances, which hold here as they are: the values of a quantised cache are exact in bf16).
Every cache is NaN, with any exponent, where no query may look."""
import math

import pytest
import torch

import paged_q8_oracle as oracle

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def spa():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_21233_amd as m
    m.load_library()
    return m


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _bytes(*shape, seed=0):
    return torch.randint(0, 256, shape, generator=torch.Generator().manual_seed(seed)).to(torch.uint8)


def _rows(*shape, seed=0):
    """bf16 rows of every size: zeros, subnormal ones, huge ones, rows with infinities and NaN, values on the borders between codes."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp2(torch.randint(-20, 21, shape[:-1] + (1,), generator=g).float())
    kind = torch.randint(0, 12, shape[:-1], generator=g)
    x[kind == 0] = 0.0
    x[kind == 1] *= 2.0 ** -120
    x[kind == 2] = torch.where(x[kind == 2] > 0, 3.0e38, 1.0e30)
    x[kind == 3] = 448.0 * torch.exp2(torch.randint(-3, 4, x[kind == 3].shape, generator=g).float())
    x[kind == 4] = torch.randint(0, 257, x[kind == 4].shape, generator=g) / 256.0          # halfway ones among them
    odd = kind == 5
    x[odd] = torch.where(torch.rand(x[odd].shape, generator=g) < 0.1, torch.tensor(math.inf), x[odd])
    x[odd] = torch.where(torch.rand(x[odd].shape, generator=g) < 0.1, torch.tensor(math.nan), x[odd])
    x[kind == 6] = -math.inf
    x[kind == 7] *= torch.exp2(torch.randint(-30, 1, x[kind == 7].shape, generator=g).float())
    return x.to(torch.bfloat16)


# --------------------------------------------------------------------------------------------------------------- append
def _slot_maps(n_pages, page):
    n = n_pages * page
    order = torch.randperm(n, generator=torch.Generator().manual_seed(n))
    yield order[:n // 2].tolist()                                  # scattered
    yield list(range(5, n - 6))                                    # one run that starts and ends inside a piece
    yield [s if s % 5 else -1 for s in range(3, n // 2)]           # padding in between
    yield [n, -1, 2 ** 31 - 1, -2 ** 31, 7]                        # outside the cache
    yield [n - 1]
    yield list(range(37, -1, -1)) + list(range(n - 40, n - 12))    # a run backwards, one forwards


def _same_codes(got, want):
    """NaN is 127 or 255"""
    got, want = got.cpu(), want
    return torch.equal(torch.where(got & 127 == 127, 127, got), torch.where(want & 127 == 127, 127, want))


def _check_append(spa, k, v, slots, cache):
    want = oracle.append_q8(k, v, torch.tensor(slots), *cache)
    mine = [x.cuda() for x in cache]
    spa.paged_append_q8(k.cuda(), v.cuda(), _i32(slots), mine[0].view(E4M3), mine[1].view(E4M3), mine[2], mine[3])
    for name, g, w in zip(("k_pages", "vt_pages"), mine, want):
        assert _same_codes(g, w), name
    assert torch.equal(mine[2].cpu(), want[2]) and torch.equal(mine[3].cpu(), want[3])


def _codes(n_pages, heads, page, head_dim):
    return [_bytes(n_pages, heads, page, head_dim, seed=1), _bytes(n_pages, heads, head_dim, page, seed=2), _bytes(n_pages, heads, page, seed=3), _bytes(n_pages, heads, page, seed=4)]


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("page,heads,n_pages", [(16, 1, 20), (32, 3, 9), (64, 8, 5), (128, 2, 7)])
def test_append_rounds_to_the_nearest(spa, head_dim, page, heads, n_pages):
    for turn, slots in enumerate(_slot_maps(n_pages, page)):
        T = len(slots)
        _check_append(spa, _rows(T, heads, head_dim, seed=turn), _rows(T, heads, head_dim, seed=50 + turn), slots, _codes(n_pages, heads, page, head_dim))


@pytest.mark.parametrize("head_dim,page,heads", [(64, 16, 2), (128, 64, 1), (128, 128, 1), (64, 32, 1)])
def test_append_of_many_tokens(spa, head_dim, page, heads):
    """Prompts that start and end anywhere, gaps, single tokens between them."""
    n_pages = 5000 // page
    n = n_pages * page
    prompts = [list(range(16 * x + x % 16, 16 * x + x % 16 + 700 + x)) for x in range(0, n // 16 - 60, 70)]
    slots = [s for p in prompts for s in p if s < n]
    slots = list(dict.fromkeys(slots))
    for x in range(40, len(slots), 97):
        slots[x] = -1
    assert len(slots) > 1500
    T = len(slots)
    _check_append(spa, _rows(T, heads, head_dim, seed=1), _rows(T, heads, head_dim, seed=2), slots, _codes(n_pages, heads, page, head_dim))
    back = slots[::-1]
    _check_append(spa, _rows(T, heads, head_dim, seed=3), _rows(T, heads, head_dim, seed=4), back, _codes(n_pages, heads, page, head_dim))


def test_append_to_strided_pages(spa):
    """K and V of one projection, pages of both and their exponents in one allocation each."""
    T, H, D, page, N = 150, 4, 128, 64, 6
    qkv = _rows(T, 3 * H, D + 16, seed=1).cuda()
    k, v = qkv[:, H:2 * H, :D], _rows(1, H, T, D, seed=2).cuda()[0].transpose(0, 1)
    both, exps = _bytes(N, 2, H, page * D, seed=3).cuda(), _bytes(N, H, 2, page, seed=4).cuda()
    cache = both[:, 0].view(N, H, page, D), both[:, 1].view(N, H, D, page), exps[:, :, 0], exps[:, :, 1]
    slots = [17 + t for t in range(T)]
    want = oracle.append_q8(k.cpu(), v.cpu(), torch.tensor(slots), *(x.cpu() for x in cache))
    spa.paged_append_q8(k, v, _i32(slots), cache[0].view(E4M3), cache[1].view(E4M3), *cache[2:])
    assert all(_same_codes(g, w) for g, w in zip(cache[:2], want)) and all(torch.equal(g.cpu(), w) for g, w in zip(cache[2:], want[2:]))


# ----------------------------------------------------------------------------------------------------------------- read
def _read_want(step, counts):
    k = torch.cat([x[:, x.shape[1] - n:].transpose(0, 1) if n <= x.shape[1] else torch.cat([x.new_zeros(x.shape[0], n - x.shape[1], x.shape[2]), x], 1).transpose(0, 1)
                   for x, n in zip(step.keys, counts)])
    v = torch.cat([x[:, x.shape[1] - n:].transpose(0, 1) if n <= x.shape[1] else torch.cat([x.new_zeros(x.shape[0], n - x.shape[1], x.shape[2]), x], 1).transpose(0, 1)
                   for x, n in zip(step.values, counts)])
    return k, v


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("page,head_dim,heads", [(16, 64, 2), (32, 128, 1), (64, 128, 3), (128, 64, 8), (16, 128, 1), (128, 128, 2)])
def test_read_gives_the_cached_tokens(spa, page, head_dim, heads, q8):
    step = oracle.Step(page, oracle.alone([0, 5, 130, 700, 64, 31], [1, 0, 3, 5, 64, 1]), page=page, head_dim=head_dim, kv_heads=heads, q8=q8)
    for counts in (step.kv_lens, [1, 0, 0, 3, 0, 1], [0, 5, 100, 333, 127, 32], [3, 9, 0, 800, 0, 40]):
        starts = [sum(counts[:b]) for b in range(len(counts) + 1)]
        rows = starts[-1] + 5
        k = torch.full((heads, rows, head_dim), 7.0, dtype=torch.bfloat16, device="cuda")
        v = torch.full((rows, heads, head_dim + 8), 7.0, dtype=torch.bfloat16, device="cuda")
        kp, vp, ke, ve = step.cache()
        spa.paged_read(kp, vp, step.table.cuda(), _i32(starts), _i32(step.kv_lens), rows, ke, ve, k=k.transpose(0, 1), v=v[:, :, :head_dim])
        want = _read_want(step, counts)
        assert torch.equal(k.transpose(0, 1)[:starts[-1]].cpu().view(torch.int16), want[0].contiguous().view(torch.int16))
        assert torch.equal(v[:starts[-1], :, :head_dim].cpu().contiguous().view(torch.int16), want[1].contiguous().view(torch.int16))
        assert (k[:, starts[-1]:] == 7.0).all() and (v[starts[-1]:] == 7.0).all() and (v[:, :, head_dim:] == 7.0).all()


def test_read_of_all_codes(spa):
    """Every code with small, large and the outermost exponents, as far as bf16 holds the value; NaN is NaN."""
    codes = torch.arange(256).to(torch.uint8).view(2, 1, 1, 128).expand(2, 1, 64, 128).contiguous()
    exps = (torch.arange(128) * 2 + 1).clamp(max=246).to(torch.uint8).view(2, 1, 64)
    table = _i32([[0, 1]])
    k, v = spa.paged_read(codes.cuda().view(E4M3), codes.transpose(2, 3).contiguous().cuda().view(E4M3), table, _i32([0, 128]), _i32([128]), 128, exps.cuda(), exps.cuda())
    want = oracle.values_of(codes, exps).transpose(1, 2).reshape(128, 1, 128)
    for x in (k, v):
        x = x.cpu().double()
        assert torch.equal(torch.isnan(x), torch.isnan(want)) and torch.equal(torch.nan_to_num(x, 0.0), torch.nan_to_num(want.to(torch.bfloat16).double(), 0.0))


# --------------------------------------------------------------------------------------------------------------- shares
def _check_shares(spa, table, starts, kv, page, least):
    got = spa.paged_shares(table.cuda(), _i32(starts), _i32(kv), page, least)
    assert torch.equal(got.cpu(), oracle.shares(table, starts, kv, page, least))


@pytest.mark.parametrize("page,batch,columns", [(16, 1, 5), (64, 2, 300), (128, 65, 40), (32, 700, 70), (16, 4096, 9), (64, 1025, 3)])
def test_shares_are_found_in_the_tables(spa, page, batch, columns):
    for seed, depth in ((1, 0.9), (2, 0.2), (3, 1.0)):
        g = torch.Generator().manual_seed(seed + batch)
        table = torch.arange(batch * columns, dtype=torch.int32).view(batch, columns)
        for b in range(1, batch):                                  # a random part of the row before
            if torch.rand((), generator=g) < depth:
                n = int(torch.randint(0, columns + 1, (), generator=g))
                table[b, :n] = table[b - 1, :n]
                if n > 3 and torch.rand((), generator=g) < 0.1:    # common again behind the first difference
                    table[b, n // 2] = -5
        new = torch.randint(0, 4, (batch,), generator=g).tolist()
        kv = [int(torch.randint(0, columns * page + 1, (), generator=g)) for _ in new]
        starts = [sum(new[:b]) for b in range(batch + 1)]
        for least in (0, 1, page * 2, 1000):
            _check_shares(spa, table, starts, kv, page, least)


def test_shares_of_special_lengths(spa):
    table = torch.tensor([[3, 4, 5]] * 6, dtype=torch.int32)
    for kv in ([192] * 6, [0] * 6, [192, 191, 129, 128, 127, 64], [193, 65, 0, 1, 66, 192], [-5, 10 ** 9, 64, 128, -1, 192]):
        _check_shares(spa, table, [0, 1, 2, 3, 3, 3, 4], [max(0, min(x, 192)) for x in kv], 64, 1)
        got = spa.paged_shares(table.cuda(), _i32([0, 1, 2, 3, 3, 3, 4]), _i32(kv), 64, 1)
        assert torch.equal(got.cpu(), oracle.shares(table, [0, 1, 2, 3, 3, 3, 4], [max(0, min(x, 192)) for x in kv], 64, 1))
    wide = torch.full((5, 12), -9, dtype=torch.int32, device="cuda")
    wide[:, 2:8] = torch.tensor([1, 2, 3, 4, 5, 6], dtype=torch.int32)
    got = spa.paged_shares(wide[:, 2:8], _i32([0, 1, 2, 3, 4, 5]), _i32([97] * 5), 16, 16)
    assert got.tolist() == [[0] * 5, [5] * 5, [80] * 5]           # the table holds 96 tokens, the last one is new: five whole pages


# ------------------------------------------------------------------------------------------------------------ attention
def _attn_close(spa, step, shared=None, lse=True, new=None, **how):
    """shared: shares to attend with, or None: paged_attn_q8"""
    call = dict(softmax_scale=how.get("scale"), n_sink_tokens=how.get("sink", 0), window_tokens=how.get("window", 0), softcap=how.get("softcap", 0.0),
                slopes=None if how.get("slopes") is None else how["slopes"].cuda(), max_new_tokens=new or 0, return_lse=lse)
    out = torch.full((step.T, *step.q.shape[1:]), 7.0, dtype=torch.bfloat16, device="cuda")
    kp, vp, ke, ve = step.cache()
    lens = step.table.cuda(), _i32(step.starts), _i32(step.kv_lens)
    if shared is None:
        got = spa.paged_attn_q8(step.q.cuda(), kp, vp, ke, ve, *lens, out=out, **call)
    else:
        got = spa.paged_attn_shared(step.q.cuda(), kp, vp, *lens, shared.cuda(), k_exp=ke, v_exp=ve, out=out, **call)
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
CHUNKS = [([0], [2]), ([5], [16]), ([64], [64]), ([100], [33]), ([0], [300]), ([1000], [129]), ([31, 700, 0], [5, 64, 130]),
          ([900, 20, 64, 0, 333], [1, 200, 1, 1, 7]), ([10, 0, 50], [0, 12, 0])]


def _q8(ctx, new, seed=None, **how):
    return oracle.Step(sum(ctx) + sum(new) if seed is None else seed, oracle.alone(ctx, new), q8=True, **how)


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("ctx", DECODE, ids=lambda c: "-".join(map(str, c))[:20])
def test_q8_attn_of_single_tokens(spa, ctx, page, head_dim):
    _attn_close(spa, _q8(ctx, [1] * len(ctx), page=page, head_dim=head_dim, padding=2, peak=2.0), new=1)


@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (8, 8), (5, 1), (10, 2), (16, 1), (17, 1), (32, 1), (33, 1), (40, 1), (70, 1), (96, 3)])
def test_q8_attn_of_head_layouts(spa, q_heads, kv_heads):
    _attn_close(spa, _q8([300, 77, 0], [1, 1, 1], q_heads=q_heads, kv_heads=kv_heads, head_dim=64), new=1)
    _attn_close(spa, _q8([300, 77, 0], [3, 40, 9], q_heads=q_heads, kv_heads=kv_heads, head_dim=64), new=40)


@pytest.mark.parametrize("head_dim,page,q_heads,kv_heads", [(128, 64, 4, 2), (64, 16, 6, 2), (128, 32, 5, 1), (64, 128, 2, 2), (128, 16, 8, 1), (64, 64, 4, 1)])
@pytest.mark.parametrize("ctx,new", CHUNKS, ids=lambda c: "-".join(map(str, c)))
def test_q8_attn_of_chunks(spa, ctx, new, head_dim, page, q_heads, kv_heads):
    step = _q8(ctx, new, page=page, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, padding=3)
    _attn_close(spa, step, new=max(new))
    _attn_close(spa, step, new=0, lse=False)


@pytest.mark.parametrize("sink,window", [(0, 1), (0, 17), (4, 1), (64, 64), (70, 100), (1, 128), (200, 33), (5000, 7), (0, 2 ** 31 - 1), (128, 300)])
@pytest.mark.parametrize("ctx,new", [([700], [1]), ([0, 63, 64, 1500, 400], [1, 1, 1, 1, 1]), ([650], [150]), ([900, 20, 300], [1, 90, 33])], ids=lambda c: "-".join(map(str, c)))
def test_q8_attn_sees_sinks_and_window_only(spa, ctx, new, sink, window):
    for page, head_dim in ((16, 64), (64, 128)):
        step = _q8(ctx, new, seed=sink % 1000 + window % 1000, page=page, head_dim=head_dim, q_heads=4, kv_heads=1)
        step.hide(sink, window)
        _attn_close(spa, step, new=max(new), sink=sink, window=window)


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("softcap,slopes", [(0.0, True), (25.0, False), (5.0, True)])
def test_q8_attn_of_every_kernel(spa, softcap, slopes, page, head_dim):
    s = torch.exp2(-torch.arange(1.0, 5.0)) if slopes else None
    for ctx, new in (([130, 0, 700], [140, 33, 1]), ([200, 33, 900], [1, 1, 2]), ([650], [90])):
        _attn_close(spa, _q8(ctx, new, q_heads=4, kv_heads=1, page=page, head_dim=head_dim, peak=2.0), new=max(new), softcap=softcap, slopes=s)


@pytest.mark.parametrize("long", [1, 40])
def test_q8_attn_over_a_long_cache(spa, long):
    step = _q8([20000, 30, 5000, 0], [long, 1, 1, 2], q_heads=4, kv_heads=1, head_dim=64, page=128)
    _attn_close(spa, step, new=long)
    _attn_close(spa, step, new=long, window=9000, sink=300)


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("q_heads", [4, 20, 40])
def test_q8_attn_of_one_long_request(spa, q_heads, head_dim):
    for ctx in (3000, 600, 511):
        step = _q8([ctx], [1], q_heads=q_heads, kv_heads=1, head_dim=head_dim, page=32)
        _attn_close(spa, step, new=1)
        _attn_close(spa, step, new=1, softcap=20.0, window=700, sink=70)


def test_q8_attn_of_rows_that_see_nothing(spa):
    for new in ([1, 1, 1], [40, 200, 7]):
        step = _q8([0, 70, 33], new, q_heads=4, kv_heads=2, page=16, head_dim=64)
        step.kv_lens = [0, new[1] - 1, 0 if new[2] == 1 else 3]
        _attn_close(spa, step, new=max(new))


@pytest.mark.parametrize("head_dim,page,q_heads", [(64, 16, 4), (128, 64, 4), (64, 128, 24)])
@pytest.mark.parametrize("ctx,new,window,sink", [(100, 1, 0, 0), (100, 4, 0, 0), (300, 7, 40, 3), (5, 150, 0, 0), (70, 150, 33, 70), (700, 130, 300, 10), (2000, 40, 0, 0)])
def test_nan_values_reach_those_who_see_them_and_no_others(spa, ctx, new, window, sink, head_dim, page, q_heads):
    step = _q8([ctx], [new], page=page, q_heads=q_heads, kv_heads=1, head_dim=head_dim)

    def call():
        kp, vp, ke, ve = step.cache()
        return spa.paged_attn_q8(step.q.cuda(), kp, vp, ke, ve, step.table.cuda(), _i32(step.starts), _i32(step.kv_lens), max_new_tokens=new,
                                 window_tokens=window, n_sink_tokens=sink).float().cpu()

    clean, n = call(), ctx + new
    odd = {n - 1: 3, n - new // 2 - 1: 9, n - new: 60, max(0, n - new - window - 1): 17, 1: 33}
    for key, dim in odd.items():
        step.vt_pages[step.table[0, key // page], 0, dim, key % page] = 127 if key % 2 else 255
    got = call()
    for i in range(new):
        pos = ctx + i
        seen = [d for j, d in odd.items() if j <= pos and (not window or pos - j < window or j < sink)]
        want = clean[i].clone()
        want[:, seen] = math.nan
        assert torch.equal(torch.isnan(got[i]), torch.isnan(want)), i
        assert torch.equal(torch.nan_to_num(got[i], 0.0), torch.nan_to_num(want, 0.0)), i


def test_q8_attn_of_strided_tensors(spa):
    step = _q8([200, 90], [1, 20], q_heads=6, kv_heads=2, page=64)
    T, N = step.T, step.k_pages.shape[0]
    kp, vp, ke, ve = step.cache()
    plain = spa.paged_attn_q8(step.q.cuda(), kp, vp, ke, ve, step.table.cuda(), _i32(step.starts), _i32(step.kv_lens))
    both = torch.empty((N, 2, 2, 64 * 128), dtype=torch.uint8, device="cuda")
    both[:, 0], both[:, 1] = kp.view(torch.uint8).flatten(2), vp.view(torch.uint8).flatten(2)
    exps = torch.stack([ke, ve], 2)
    room = torch.full((6, T, 160), 7.0, dtype=torch.bfloat16, device="cuda")
    got = spa.paged_attn_q8(step.q.cuda(), both[:, 0].view(N, 2, 64, 128).view(E4M3), both[:, 1].view(N, 2, 128, 64).view(E4M3), exps[:, :, 0], exps[:, :, 1],
                            step.table.cuda(), _i32(step.starts), _i32(step.kv_lens), out=room[:, :, 16:144].transpose(0, 1))
    assert torch.equal(got.view(torch.int16), plain.view(torch.int16))
    assert (room[:, :, :16] == 7.0).all() and (room[:, :, 144:] == 7.0).all()


# -------------------------------------------------------------------------------------------------------- shared prompts
GROUPS = {
    "decode": [(700, [(0, 1), (5, 1), (130, 1)])],
    "none": [(0, [(100, 1)]), (0, [(0, 3)])],
    "two": [(300, [(10, 1), (0, 2)]), (0, [(90, 1)]), (1500, [(3, 1), (64, 1), (200, 4), (0, 1)])],
    "many": [(640, [(b % 7 * 20, 1) for b in range(70)]), (200, [(b, 1) for b in range(5)])],
    "chunks": [(400, [(20, 90), (0, 1), (77, 33)]), (130, [(0, 60), (1, 60)])],
    "short": [(64, [(0, 1), (1, 1)]), (128, [(0, 1)] * 3)],
    "long": [(9000, [(100, 1), (0, 1), (63, 1), (2, 3)]), (3000, [(40, 1), (40, 1)])],
}


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("page,head_dim,q_heads,kv_heads", [(16, 64, 4, 1), (64, 128, 4, 2), (32, 128, 8, 1), (128, 64, 6, 2)])
@pytest.mark.parametrize("groups", GROUPS, ids=list(GROUPS))
def test_shared_attn_of_groups(spa, groups, page, head_dim, q_heads, kv_heads, q8):
    step = oracle.Step(len(groups) + page, GROUPS[groups], page=page, head_dim=head_dim, q_heads=q_heads, kv_heads=kv_heads, q8=q8, padding=3, peak=2.0)
    _attn_close(spa, step, shared=step.shares, new=max(step.new))
    _attn_close(spa, step, shared=step.shares, lse=False)
    found = spa.paged_shares(step.table.cuda(), _i32(step.starts), _i32(step.kv_lens), page, 1)
    _attn_close(spa, step, shared=found.cpu(), new=max(step.new))


@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (8, 8), (5, 1), (16, 1), (17, 1), (33, 1), (70, 1), (96, 3)])
def test_shared_attn_of_head_layouts(spa, q_heads, kv_heads):
    for q8 in (False, True):
        step = oracle.Step(q_heads, [(300, [(4, 1), (70, 1), (0, 1)]), (200, [(1, 5), (0, 30)])], q_heads=q_heads, kv_heads=kv_heads, head_dim=64, q8=q8)
        _attn_close(spa, step, shared=step.shares, new=30)


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("sink,window", [(0, 1), (0, 17), (4, 1), (64, 64), (70, 100), (500, 33), (5000, 7), (0, 2 ** 31 - 1), (128, 600), (3, 1400)])
@pytest.mark.parametrize("groups", ["two", "chunks", "long"])
def test_shared_attn_sees_sinks_and_window_only(spa, groups, sink, window, q8):
    step = oracle.Step(sink + window % 1000, GROUPS[groups], page=64, head_dim=64, q_heads=4, kv_heads=1, q8=q8)
    if window < 10000:
        step.hide(sink, window)
    _attn_close(spa, step, shared=step.shares, new=max(step.new), sink=sink, window=window)


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("head_dim,page", [(64, 16), (128, 32), (64, 64), (128, 64)])
@pytest.mark.parametrize("softcap,slopes", [(0.0, True), (25.0, False), (5.0, True)])
def test_shared_attn_with_capped_logits_and_bias_by_distance(spa, softcap, slopes, head_dim, page, q8):
    s = torch.exp2(-torch.arange(1.0, 5.0)) if slopes else None
    for groups in ("two", "chunks", "many"):
        step = oracle.Step(7, GROUPS[groups], page=page, head_dim=head_dim, q_heads=4, kv_heads=1, q8=q8, peak=2.0)
        _attn_close(spa, step, shared=step.shares, new=max(step.new), softcap=softcap, slopes=s)


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_shared_attn_of_requests_left_out(spa, q8):
    """Requests without tokens or without keys inside a group change nothing for the others and get zeros."""
    step = oracle.Step(3, [(640, [(5, 1), (0, 0), (9, 1), (70, 3)]), (300, [(0, 1), (33, 2)])], q_heads=4, kv_heads=2, head_dim=64, q8=q8, padding=2)
    _attn_close(spa, step, shared=step.shares, new=3)
    step.kv_lens[2] = 0
    step.kv_lens[5] = 1
    _attn_close(spa, step, shared=step.shares, new=3)
    step.kv_lens[0] = 100                                          # the first of the group has less than the others have in common
    _attn_close(spa, step, shared=step.shares, new=3)


@pytest.mark.parametrize("tokens", [1, 63, 64, 100, 640, 641])
def test_shared_attn_of_any_common_length(spa, tokens):
    """Fewer tokens than the requests have in common pages, or more than whole tiles."""
    step = oracle.Step(3, [(640, [(5, 1), (0, 1), (9, 2)])], page=16, q_heads=4, kv_heads=2, head_dim=64, q8=True)
    step.shares[2] = tokens
    _attn_close(spa, step, shared=step.shares, new=2)


def test_shared_attn_of_many_requests(spa):
    groups = [(64 * (x % 5) + 100, [((7 * b + x) % 90, 1 + (b % 50 == 7) * 30) for b in range(1 + 13 * x % 37)]) for x in range(30)]
    for q8 in (False, True):
        step = oracle.Step(300, groups, q_heads=2, kv_heads=1, head_dim=64, page=32, q8=q8)
        _attn_close(spa, step, shared=step.shares, new=31)
