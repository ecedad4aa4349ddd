"""Edges of the paged KV cache on the GPU: how exact a few rows' attention is, values that are not finite, calls that are cut, lists of
slots long enough for the append kernel of prompts, malformed lengths next to memory that must not change.  Against the plain 64-bit forms
of tests/paged_oracle.py."""
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


def _attn(spa, step, **how):
    return spa.paged_attn(step.q.cuda(), step.k_pages.cuda(), step.vt_pages.cuda(), step.table.cuda(), _i32(step.starts), _i32(step.kv_lens), **how)


# ------------------------------------------------------------------------------------- weights of few rows keep 16 bits
def _within_the_output_s_rounding(step, out, rows):
    """The oracle's tolerance with another share for the weights: two bf16 parts leave a rest of 2^-8 of 2^-8 of a weight, and the sum of
    n products in fp32 takes at most 2^-23 of their sizes a term (half a step, or a whole one where the matrix unit cuts off)."""
    want, _, tol, _ = step.want()
    mass = oracle.attn(step.q, step.keys, [v.abs() for v in step.values], step.starts, step.kv_lens)[0]
    n = max(step.kv_lens)
    tol = tol - 1.01 * 2 ** -8 * mass + (1.01 * 2 ** -16 + (n + 8) * 2 ** -23) * mass
    off = (out.cpu().double() - want).abs() - tol
    assert off[rows].max().item() <= 0, (off[rows].max().item(), (off == off[rows].max()).nonzero()[0].tolist())


@pytest.mark.parametrize("head_dim,page,q_heads,kv_heads", [(128, 64, 4, 1), (64, 16, 8, 2), (128, 16, 16, 1), (128, 32, 20, 1), (64, 128, 32, 1)])
@pytest.mark.parametrize("batch", [1, 5, 90])
def test_single_tokens_are_as_exact_as_the_output_type(spa, batch, head_dim, page, q_heads, kv_heads):
    """Few and many requests, 16 and 32 rows a workgroup: every kernel for few rows."""
    g = torch.Generator().manual_seed(batch)
    ctx = torch.randint(0, 120, (batch,), generator=g).tolist()
    step = oracle.Step(batch + page, ctx, [1] * batch, page=page, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim)
    _within_the_output_s_rounding(step, _attn(spa, step, max_new_tokens=1), slice(None))


def test_single_tokens_next_to_a_chunk_are_as_exact_as_the_output_type(spa):
    step = oracle.Step(7, [60, 40, 3, 100], [1, 2, 70, 4], q_heads=4, kv_heads=1)
    rows = [t for b in (0, 1, 3) for t in range(step.starts[b], step.starts[b + 1])]
    _within_the_output_s_rounding(step, _attn(spa, step, max_new_tokens=70), rows)


def test_cut_key_axes_are_as_exact_as_the_output_type(spa):
    """700 keys in pieces of four tiles and their merge."""
    step = oracle.Step(8, [700], [1], q_heads=4, kv_heads=1)
    _within_the_output_s_rounding(step, _attn(spa, step, max_new_tokens=1), slice(None))


@pytest.mark.parametrize("q_heads", [4, 20])
def test_infinite_values_with_weights_of_one_part(spa, q_heads):
    """A weight of 1 has nothing left for its second part: 0 times an infinite value must not show."""
    step = oracle.Step(1, [0, 0, 0, 0], [1, 1, 1, 1], q_heads=q_heads, kv_heads=1, head_dim=64)
    for b, value in enumerate((math.inf, -math.inf, math.nan)):
        step.vt_pages[step.table[b, 0], 0, 5, 0] = value
    got, values = _attn(spa, step).float().cpu(), torch.stack([v[0, 0] for v in step.values]).float()
    values[:3, 5] = torch.tensor([math.inf, -math.inf, math.nan])
    assert torch.equal(got.nan_to_num(7e9), values[:, None].expand_as(got).nan_to_num(7e9))


# ------------------------------------------------------------------------------------------- pieces of a cut key axis
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_values_that_are_not_finite_in_a_piece_without_weight(spa, value, new):
    """The bias leaves the first keys' piece a weight of 2^-2000 of the last one's, nothing in fp32."""
    step = oracle.Step(3, [3000], [new], q_heads=4, kv_heads=1, head_dim=64)
    slopes = torch.full((4,), 0.5, device="cuda")
    clean = _attn(spa, step, max_new_tokens=new, slopes=slopes).float().cpu()
    step.vt_pages[step.table[0, 0], 0, 7, 5] = value
    got = _attn(spa, step, max_new_tokens=new, slopes=slopes).float().cpu()
    odd = got[:, :, 7]
    assert (torch.isnan(odd) | (odd == value)).all()
    got[:, :, 7] = clean[:, :, 7]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("ctx,new", [(100, 1), (100, 40), (3000, 1), (3000, 40)])
def test_keys_with_logits_of_minus_infinity(spa, ctx, new):
    """Weights of 0 next to other keys, also where a whole piece has them; where a query sees no other key its output is NaN, and still zeros
    where it sees none at all."""
    step = oracle.Step(5, [ctx, ctx], [new, new], q_heads=4, kv_heads=1, head_dim=64)
    step.q[:, :, 0] = 1.0
    for b, upto in ((0, step.kv_lens[0] // 2), (1, step.kv_lens[1])):
        step.keys[b][:, :upto, 0] = -math.inf
        for key in range(upto):
            step.k_pages[step.table[b, key // step.page], 0, key % step.page, 0] = -math.inf
    out, lse = _attn(spa, step, max_new_tokens=new, return_lse=True)
    want, want_lse, tol, lse_tol = oracle.attn(step.q[:new], step.keys[:1], step.values[:1], [0, new], step.kv_lens[:1])
    assert ((out[:new].cpu().double() - want).abs() <= tol).all() and ((lse[:new].cpu().double() - want_lse).abs() <= lse_tol).all()
    assert torch.isnan(out[new:]).all() and (lse[new:] == -math.inf).all()
    step.kv_lens[1] = new - 1                                       # the first new token has no position
    out, lse = _attn(spa, step, max_new_tokens=new, return_lse=True)
    assert (out[new] == 0).all() and torch.isnan(out[new + 1:]).all() and (lse[new:] == -math.inf).all()


# ------------------------------------------------------------------------------------------------ arrays in one tensor
def test_queries_and_outputs_as_slices_of_one_tensor(spa):
    """out in the place of the keys that the step has appended, next to its own queries; on them it is refused."""
    step = oracle.Step(6, [90, 10, 400], [1, 40, 2], q_heads=4, kv_heads=2, head_dim=64)
    qkv = torch.full((step.T, 12, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    qkv[:, :4] = step.q.cuda()
    t = step.k_pages.cuda(), step.vt_pages.cuda(), step.table.cuda(), _i32(step.starts), _i32(step.kv_lens)
    want = spa.paged_attn(step.q.cuda(), *t)
    got = spa.paged_attn(qkv[:, :4], *t, out=qkv[:, 4:8])
    assert torch.equal(got, want) and torch.equal(qkv[:, 4:8], want) and (qkv[:, 8:] == 7.0).all() and torch.equal(qkv[:, :4].cpu(), step.q)
    for h in (0, 1, 3):
        with pytest.raises(spa.SpaError):
            spa.paged_attn(qkv[:, :4], *t, out=qkv[:, h:h + 4])
    with pytest.raises(spa.SpaError):
        spa.paged_attn(qkv[1:, :4], *t, out=qkv[:-1, :4])


# --------------------------------------------------------------------------- append: the kernel for more than 1024 tokens
def _bits(*shape, seed=0):
    """bf16 values of any bits, NaN payloads among them"""
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-2 ** 15, 2 ** 15, shape, generator=g).to(torch.int16).view(torch.bfloat16)


def _same_bits(a, b):
    return torch.equal(a.cpu().view(torch.int16), b.cpu().view(torch.int16))


def _prompts(T, n_pages, page, seed):
    """Slots of prompts whose first and last tokens lie inside pages, the pages in any order; padding behind them."""
    g = torch.Generator().manual_seed(seed)
    draw = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=g))  # noqa: E731
    ids, slots = torch.randperm(n_pages, generator=g).tolist(), []
    while len(slots) < T:
        ctx, n = draw(0, 2 * page), min(draw(1, 500), T - len(slots))
        pages = [ids.pop() for _ in range(-(-(ctx % page + n) // page))]
        slots += [pages[(ctx % page + i) // page] * page + (ctx % page + i) % page for i in range(n)]
        if len(slots) < T and draw(0, 3) == 0:
            slots.append(-1)
    return slots


def _long_slot_maps(T, n_pages, page):
    n = n_pages * page
    yield "scattered", torch.randperm(n, generator=torch.Generator().manual_seed(T)).tolist()[:T]
    for start in (0, 1, 4, 7):                                     # a piece begins at token 0, 7, 4, 1 and every 8th from there, over the borders of 64
        yield f"one run from {start}", list(range(start, start + T))
    yield "prompts", _prompts(T, n_pages, page, T)
    yield "gaps", [s if (s + 3) % 13 else -1 for s in range(2, T + 2)]
    yield "backwards", list(range(T - 1, -1, -1))
    yield "wild", [(n + s, -1 - s, 2 ** 31 - 1 - s, s)[s % 4] if s % 64 > 50 else s for s in range(T)]
    yield "swapped pairs", [s ^ 1 for s in range(T + 1)][:T]


@pytest.mark.parametrize("T", [1024, 1025, 1087, 3101])
@pytest.mark.parametrize("head_dim,page,heads", [(64, 16, 3), (128, 32, 1), (128, 64, 2), (64, 128, 1)])
def test_append_of_many_tokens_moves_the_bits(spa, head_dim, page, heads, T):
    n_pages = 2 * T // page + 40
    k_pages, vt_pages = _bits(n_pages, heads, page, head_dim, seed=90), _bits(n_pages, heads, head_dim, page, seed=91)
    for turn, (name, slots) in enumerate(_long_slot_maps(T, n_pages, page)):
        k, v = _bits(T, heads, head_dim, seed=turn), _bits(T, heads, head_dim, seed=50 + turn)
        want = oracle.append(k, v, torch.tensor(slots), k_pages, vt_pages)
        mine = k_pages.cuda(), vt_pages.cuda()
        spa.paged_append(k.cuda(), v.cuda(), _i32(slots), *mine)
        assert _same_bits(mine[0], want[0]) and _same_bits(mine[1], want[1]), name


def test_append_of_many_strided_tokens(spa):
    """K and V out of one projection's output and out of [heads, tokens, dim]; pages of both in one allocation, with room between them."""
    T, H, D, page, N = 1500, 3, 128, 32, 60
    qkv, v = _bits(T, 4 * H, D + 8, seed=1).cuda(), _bits(H, T, D, seed=2).cuda().transpose(0, 1)
    both = _bits(N, 5, H, page * D, seed=3).cuda()
    before = both.clone()
    k_pages, vt_pages = both[:, 1].view(N, H, page, D), both[:, 3].view(N, H, D, page)
    slots = _prompts(T, N, page, 9)
    want = oracle.append(qkv[:, H:2 * H, :D].cpu(), v.cpu(), torch.tensor(slots), k_pages.cpu(), vt_pages.cpu())
    spa.paged_append(qkv[:, H:2 * H, :D], v, _i32(slots), k_pages, vt_pages)
    assert _same_bits(k_pages, want[0]) and _same_bits(vt_pages, want[1])
    assert all(_same_bits(both[:, i], before[:, i]) for i in (0, 2, 4))


def test_append_of_many_tokens_far_past_32_bit_offsets(spa):
    page, H, D, T = 128, 1, 128, 1300
    n_pages = 5 * 2 ** 30 // (page * H * D * 2)
    k_pages = torch.zeros((n_pages, H, page, D), dtype=torch.bfloat16, device="cuda")
    vt_pages = torch.zeros((n_pages, H, D, page), dtype=torch.bfloat16, device="cuda")
    k, v = _bits(T, H, D, seed=1), _bits(T, H, D, seed=2)
    first = n_pages * page - T - 3                                  # up to the third last slot of the cache
    spa.paged_append(k.cuda(), v.cuda(), _i32(list(range(first, first + T))), k_pages, vt_pages)
    at = first // page
    got_k = k_pages[at:].transpose(1, 2).reshape(-1, H, D)
    got_v = vt_pages[at:].permute(0, 3, 1, 2).reshape(-1, H, D)
    skip = first - at * page
    for got, x in ((got_k, k), (got_v, v)):
        assert _same_bits(got[skip:skip + T], x) and (got[:skip] == 0).all() and (got[skip + T:] == 0).all()
    assert (k_pages[:at] == 0).all() and (vt_pages[:at] == 0).all()


# --------------------------------------------------------------------------------- malformed lengths, next to other memory
MALFORMED = [[0, 1, 2, 10 ** 9], [-5, 1, 2, 3], [0, 3, 1, 3], [2, 1, 0, 0], [0, 2 ** 31 - 1, -2 ** 31, 3], [0, 48, 0, 48], [48, 0, 48, 0]]


@pytest.mark.parametrize("max_new", [0, 1, 48])
@pytest.mark.parametrize("head_dim,q_heads", [(64, 4), (128, 20)])
def test_malformed_lengths_of_calls_that_are_cut_change_nothing_around(spa, head_dim, q_heads, max_new):
    """out, lse and workspace lie inside larger buffers: what is around them keeps its bits, for few and for many rows, in pieces and merged;
    with sound starts the other requests are right whatever one request's length is."""
    step = oracle.Step(2, [2600, 2400, 1900], [1, 40, 7], q_heads=q_heads, kv_heads=1, head_dim=head_dim, page=32)
    T, Hq, D = step.q.shape
    t = step.q.cuda(), step.k_pages.cuda(), step.vt_pages.cuda(), step.table.cuda()
    n_pages, C, page = t[1].shape[0], t[3].shape[1], 32
    p = spa.make_paged_params(batch=3, n_q_heads=Hq, n_kv_heads=1, head_dim=D, page_size=page, n_pages=n_pages, max_pages=C, n_tokens=T,
                              max_new_tokens=max_new, table_stride=C, q=(Hq * D, D), out=(Hq * D, D), k_pages=(page * D, page * D),
                              vt_pages=(page * D, page * D))
    ws_bytes = spa.paged_workspace_bytes(p)
    assert ws_bytes > 0
    sizes = T * Hq * D * 2, T * Hq * 4, ws_bytes
    margin = 1 << 16
    want, want_lse, tol, lse_tol = step.want()
    for starts, kv in [(s, step.kv_lens) for s in MALFORMED] + [(step.starts, [step.kv_lens[0], x, step.kv_lens[2]]) for x in (10 ** 9, -5, 0)]:
        room = [torch.full((2 * margin + n,), 0xa5, dtype=torch.uint8, device="cuda") for n in sizes]
        at = [x.data_ptr() + margin for x in room]
        q_starts, kv_lens = _i32(starts), _i32(kv)
        rc = spa.load_library().sparse_prefill_paged_attn(bytes(p), t[0].data_ptr(), t[1].data_ptr(), t[2].data_ptr(), t[3].data_ptr(), q_starts.data_ptr(),
                                                          kv_lens.data_ptr(), None, at[0], at[1], at[2], ws_bytes, torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        for x, n in zip(room, sizes):
            assert (x[:margin] == 0xa5).all() and (x[margin + n:] == 0xa5).all(), (starts, kv)
        if starts == step.starts:
            out = room[0][margin:margin + sizes[0]].view(torch.bfloat16).view(T, Hq, D).cpu().double()
            lse = room[1][margin:margin + sizes[1]].view(torch.float32).view(T, Hq).cpu().double()
            rows = [0] + list(range(step.starts[2], T))
            assert ((out - want).abs() <= tol)[rows].all() and ((lse - want_lse).abs() <= lse_tol)[rows].all()


@pytest.mark.parametrize("T", [60, 1500])
def test_append_to_slots_that_occur_twice_leaves_values_of_their_tokens(spa, T):
    """Each value one of the tokens' own, whichever; nothing else changes."""
    N, H, D, page = 60, 2, 64, 32
    half = T // 2
    for again in (list(range(3, 3 + half)), list(range(10, 10 + half)), list(range(2 + half, 2, -1))):
        slots = list(range(3, 3 + half)) + again
        k, v = _bits(T, H, D, seed=1), _bits(T, H, D, seed=2)
        k_pages, vt_pages = _bits(N, H, page, D, seed=3), _bits(N, H, D, page, seed=4)
        first = oracle.append(k, v, torch.tensor(slots), k_pages, vt_pages)
        last = oracle.append(k.flip(0), v.flip(0), torch.tensor(slots).flip(0), k_pages, vt_pages)
        mine = k_pages.cuda(), vt_pages.cuda()
        spa.paged_append(k.cuda(), v.cuda(), _i32(slots), *mine)
        for got, a, b in zip(mine, first, last):
            got, a, b = (x.cpu().view(torch.int16) for x in (got, a, b))
            assert ((got == a) | (got == b)).all()


def test_append_to_more_pages_than_a_field_holds_is_refused(spa):
    k_pages = torch.zeros((1, 1, 16, 64), dtype=torch.bfloat16, device="cuda").expand(2 ** 31, 1, 16, 64)
    vt_pages = torch.zeros((1, 1, 64, 16), dtype=torch.bfloat16, device="cuda").expand(2 ** 31, 1, 64, 16)
    x = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(spa.SpaError):
        spa.paged_append(x, x, _i32([0]), k_pages, vt_pages)
