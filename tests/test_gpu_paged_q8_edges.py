"""Edges of the quantised paged cache and of shared prompts on the GPU: how exact few rows are, values that are not finite, malformed inputs next to
memory that must not change, caches past 4 GiB, captured steps, streams, and the calls one after the other as a program makes them."""
import math

import pytest
import torch

import paged_oracle
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


def _attn(spa, step, shares=None, **how):
    kp, vp, ke, ve = step.cache()
    lens = step.table.cuda(), _i32(step.starts), _i32(step.kv_lens)
    if shares is None:
        return spa.paged_attn_q8(step.q.cuda(), kp, vp, ke, ve, *lens, **how)
    return spa.paged_attn_shared(step.q.cuda(), kp, vp, *lens, shares.cuda(), k_exp=ke, v_exp=ve, **how)


# ------------------------------------------------------------------------------------- weights of few rows keep 16 bits
def _within_the_output_s_rounding(step, out, rows):
    """The oracle's tolerance with another share for the weights: two bf16 parts leave a rest of 2^-8 of 2^-8 of a weight, and the sum of
    n products in fp32 takes at most 2^-23 of their sizes a term (half a step, or a whole one where the matrix unit cuts off)."""
    want, _, tol, _ = step.want()
    mass = paged_oracle.attn(step.q, step.keys, [v.abs() for v in step.values], step.starts, step.kv_lens)[0]
    n = max(step.kv_lens)
    tol = tol - 1.01 * 2 ** -8 * mass + (1.01 * 2 ** -16 + (n + 8) * 2 ** -23) * mass
    off = (out.cpu().double() - want).abs() - tol
    assert off[rows].max().item() <= 0, (off[rows].max().item(), (off == off[rows].max()).nonzero()[0].tolist())


@pytest.mark.parametrize("head_dim,page,q_heads,kv_heads", [(128, 64, 4, 1), (64, 16, 8, 2), (128, 16, 16, 1), (128, 32, 20, 1), (64, 128, 32, 1), (64, 32, 4, 1)])
@pytest.mark.parametrize("batch", [1, 5, 90])
def test_single_tokens_are_as_exact_as_the_output_type(spa, batch, head_dim, page, q_heads, kv_heads):
    g = torch.Generator().manual_seed(batch)
    ctx = torch.randint(0, 120, (batch,), generator=g).tolist()
    step = oracle.Step(batch + page, oracle.alone(ctx, [1] * batch), page=page, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, q8=True)
    _within_the_output_s_rounding(step, _attn(spa, step, max_new_tokens=1), slice(None))


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_few_rows_with_a_shared_prompt_are_as_exact_as_the_output_type(spa, q8):
    """16 rows of a group, and its requests' own keys: two parts and more, joined."""
    step = oracle.Step(8, [(700, [(5, 1), (90, 1), (0, 1), (33, 1)])], q_heads=4, kv_heads=1, q8=q8)
    _within_the_output_s_rounding(step, _attn(spa, step, shares=step.shares, max_new_tokens=1), slice(None))


# ------------------------------------------------------------------------------------------- values that are not finite
@pytest.mark.parametrize("new", [1, 40])
def test_nan_in_a_piece_without_weight(spa, new):
    """The bias leaves the first keys' piece a weight of 2^-2000 of the last one's, nothing in fp32."""
    step = oracle.Step(3, oracle.alone([3000], [new]), q_heads=4, kv_heads=1, head_dim=64, q8=True)
    slopes = torch.full((4,), 0.5, device="cuda")
    clean = _attn(spa, step, max_new_tokens=new, slopes=slopes).float().cpu()
    step.vt_pages[step.table[0, 0], 0, 7, 5] = 127
    got = _attn(spa, step, max_new_tokens=new, slopes=slopes).float().cpu()
    assert torch.isnan(got[:, :, 7]).all()
    got[:, :, 7] = clean[:, :, 7]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("new", [1, 70])
def test_a_nan_key_reaches_those_who_see_it(spa, new):
    step = oracle.Step(5, oracle.alone([100, 100, 300], [new, 1, 1]), q_heads=2, kv_heads=1, head_dim=64, q8=True)
    clean = _attn(spa, step)
    at = 100 + new // 2
    step.k_pages[step.table[0, at // 64], 0, at % 64, 9] = 255
    got = _attn(spa, step)
    assert torch.isnan(got[new // 2:new]).all()
    assert torch.equal(got[:new // 2], clean[:new // 2]) and torch.equal(got[new:], clean[new:])


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("requests,window,sink", [([(5, 1), (90, 1), (0, 1)], 0, 0), ([(5, 3), (90, 40), (0, 2)], 0, 0), ([(70, 30), (300, 5)], 250, 3), ([(0, 1)] * 40, 100, 70)])
def test_values_that_are_not_finite_under_a_shared_prompt(spa, requests, window, sink, q8):
    step = oracle.Step(len(requests), [(320, requests)], q_heads=4, kv_heads=1, head_dim=64, q8=q8)
    how = dict(shares=step.shares, window_tokens=window, n_sink_tokens=sink)
    clean = _attn(spa, step, **how).float().cpu()
    B = len(requests)
    odd = [(0, 3, 5, math.nan), (0, 319, 9, math.nan if q8 else math.inf), (0, 200, 60, math.nan if q8 else -math.inf)]      # (request, key, dim): of all
    odd += [(b, step.kv_lens[b] - 1, 20 + b % 3, math.nan) for b in range(0, B, 2)]
    for b, key, dim, value in odd:
        step.vt_pages[step.table[b, key // 64], 0, dim, key % 64] = 127 if q8 else value
    got = _attn(spa, step, **how).float().cpu()
    for b, (_, new) in enumerate(requests):
        for i in range(new):
            pos = step.kv_lens[b] - new + i
            want = clean[step.starts[b] + i].clone()
            for owner, key, dim, value in odd:
                if (owner == b or key < 320) and key <= pos and (not window or pos - key < window or key < sink):
                    want[:, dim] = value
            assert torch.equal(got[step.starts[b] + i].nan_to_num(7e9), want.nan_to_num(7e9)), (b, i)


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("sink,window", [(0, 100), (70, 300), (5, 1)])
def test_a_request_left_out_does_not_cut_the_others_window(spa, sink, window, q8):
    """Rows of requests without keys, or with fewer than the group has in common, lie in one tile with others."""
    step = oracle.Step(3, [(640, [(5, 1), (0, 2), (9, 1), (70, 30)])], q_heads=4, kv_heads=2, head_dim=64, q8=q8)
    for b, kv in ((2, 0), (1, 200), (0, 3)):
        step.kv_lens[b] = kv
        how = dict(sink=sink, window=window)
        want, _, tol, _ = step.want(**how)
        got = _attn(spa, step, shares=step.shares, n_sink_tokens=sink, window_tokens=window)
        assert ((got.cpu().double() - want).abs() - tol).max().item() <= 0


# ----------------------------------------------------------------------------------------------------- malformed inputs
def _guarded(shape, dtype, fill):
    """A tensor in the middle of an allocation whose rest must not change."""
    n = math.prod(shape)
    whole = torch.full((3 * n + 4096,), fill, dtype=dtype, device="cuda")
    return whole, whole[n + 2048 - n % 16:][:n].view(shape)


def _around(whole, inner):
    first = (inner.data_ptr() - whole.data_ptr()) // whole.element_size()
    return torch.cat([whole[:first], whole[first + inner.numel():]])


WILD = [2 ** 31 - 1, -2 ** 31, -1, 0, 1, 2, 7, 10 ** 9, 64, 65]


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_wild_shares_lengths_and_tables_change_nothing_around(spa, q8):
    g = torch.Generator().manual_seed(5)
    step = oracle.Step(6, [(300, [(10, 1), (0, 2), (70, 30)]), (0, [(90, 1)])], q_heads=8, kv_heads=2, head_dim=64, page=16, q8=q8)
    kp, vp, ke, ve = step.cache()
    T, B = step.T, 4
    wild = lambda *s: torch.tensor(WILD, dtype=torch.int32)[torch.randint(0, len(WILD), s, generator=g)].cuda()  # noqa: E731
    whole_out, out = _guarded((T, 8, 64), torch.bfloat16, 7.0)
    need = 0
    for turn in range(40):
        shares = wild(3, B) if turn % 4 else step.shares.cuda()
        table = wild(*step.table.shape) if turn % 3 == 0 else step.table.cuda()
        starts = wild(B + 1) if turn % 5 == 1 else _i32(step.starts)
        kv = wild(B) if turn % 5 == 2 else _i32(step.kv_lens)
        ws = None
        if turn % 2:
            if not need:
                need = spa.paged_shared_workspace_bytes(spa.make_paged_params(
                    batch=B, n_q_heads=8, n_kv_heads=2, head_dim=64, page_size=16, n_pages=kp.shape[0], max_pages=table.shape[1], n_tokens=T,
                    table_stride=table.shape[1]))
            whole_ws = torch.full((need + 8192,), 255, dtype=torch.uint8, device="cuda")        # NaN in the places of partial results
            at = 4096 - (whole_ws.data_ptr() + 4096) % 256 + 256
            ws = whole_ws[at:at + need]
        spa.paged_attn_shared(step.q.cuda(), kp, vp, table, starts, kv, shares, k_exp=ke, v_exp=ve, out=out, workspace=ws, return_lse=turn % 2 == 0)
        torch.cuda.synchronize()
        assert (_around(whole_out, out) == 7.0).all()
        if ws is not None:
            assert (_around(whole_ws, ws) == 255).all()
        spa.paged_shares(table, starts, kv, 16, 1)
    want = _attn(spa, step, shares=step.shares)
    spa.paged_attn_shared(step.q.cuda(), kp, vp, step.table.cuda(), _i32(step.starts), _i32(step.kv_lens), step.shares.cuda(), k_exp=ke, v_exp=ve, out=out)
    assert torch.equal(out.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_read_of_wild_lengths_and_tables_changes_nothing_around(spa, q8):
    g = torch.Generator().manual_seed(6)
    step = oracle.Step(7, oracle.alone([100, 33, 0], [1, 2, 3]), kv_heads=2, head_dim=64, page=16, q8=q8)
    kp, vp, ke, ve = step.cache()
    wild = lambda *s: torch.tensor(WILD, dtype=torch.int32)[torch.randint(0, len(WILD), s, generator=g)].cuda()  # noqa: E731
    n = 150
    whole_k, k = _guarded((n, 2, 64), torch.bfloat16, 7.0)
    whole_v, v = _guarded((n, 2, 64), torch.bfloat16, 7.0)
    for turn in range(30):
        table = wild(*step.table.shape) if turn % 3 == 0 else step.table.cuda()
        starts = wild(4) if turn % 3 == 1 else _i32([0, 101, 136, 139])
        kv = wild(3) if turn % 3 == 2 else _i32(step.kv_lens)
        spa.paged_read(kp, vp, table, starts, kv, n, ke, ve, k=k, v=v)
        torch.cuda.synchronize()
        assert (_around(whole_k, k) == 7.0).all() and (_around(whole_v, v) == 7.0).all()


def test_quantised_attention_of_wild_lengths_and_tables_leaves_others_alone(spa):
    step = oracle.Step(6, oracle.alone([100, 50, 80], [1, 1, 1]), q_heads=4, kv_heads=1, head_dim=64, q8=True)
    kp, vp, ke, ve = step.cache()
    call = lambda table, starts, kv, **how: spa.paged_attn_q8(step.q.cuda(), kp, vp, ke, ve, table.cuda(), _i32(starts), _i32(kv), **how)  # noqa: E731
    clean = call(step.table, step.starts, step.kv_lens)
    table = step.table.clone()
    table[1] = torch.tensor([2 ** 31 - 1, -2 ** 31])
    for kv in ([101, 10 ** 9, 81], [101, -5, 81], [101, 2 ** 31 - 1, 81]):
        got = call(table, step.starts, kv)
        assert torch.equal(got[0], clean[0]) and torch.equal(got[2], clean[2])
    for starts in ([0, 1, 2, 10 ** 9], [-5, 1, 2, 3], [0, 3, 1, 3], [2, 1, 0, 0], [0, 2 ** 31 - 1, -2 ** 31, 3]):
        call(step.table, starts, step.kv_lens, max_new_tokens=1)
        call(step.table, starts, step.kv_lens)
    torch.cuda.synchronize()


def test_a_quantised_cache_far_past_32_bit_offsets(spa):
    """Pages behind the first 4 GiB."""
    page, H, D = 128, 1, 128
    n_pages = 5 * 2 ** 30 // (page * H * D)
    step = oracle.Step(8, oracle.alone([700], [1]), page=page, q_heads=2, kv_heads=H, head_dim=D, q8=True)
    k = torch.zeros((n_pages, H, page, D), dtype=torch.uint8, device="cuda")
    vt = torch.zeros((n_pages, H, D, page), dtype=torch.uint8, device="cuda")
    ke, ve = torch.ones((2, n_pages, H, page), dtype=torch.uint8, device="cuda")
    table = step.table.clone()
    for j in range(table.shape[1]):
        there = n_pages - 1 - 3 * j
        for big, small in ((k, step.k_pages), (vt, step.vt_pages), (ke, step.k_exp), (ve, step.v_exp)):
            big[there] = small[table[0, j]].cuda()
        table[0, j] = there
    near = _attn(spa, step)
    far = spa.paged_attn_q8(step.q.cuda(), k.view(E4M3), vt.view(E4M3), ke, ve, table.cuda(), _i32(step.starts), _i32(step.kv_lens))
    assert torch.equal(near, far)
    rk, rv = spa.paged_read(k.view(E4M3), vt.view(E4M3), table.cuda(), _i32([0, 701]), _i32([701]), 701, ke, ve)
    assert torch.equal(rk.cpu(), step.keys[0].transpose(0, 1)) and torch.equal(rv.cpu(), step.values[0].transpose(0, 1))
    x = torch.randn(1500, H, D, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    codes, e = oracle.quantise(x)
    for n in (3, 1500):                                            # both kernels
        slots = [n_pages * page - 1 - t if n == 3 else (n_pages - 20) * page + t for t in range(n)]
        spa.paged_append_q8(x[:n].cuda(), x[:n].cuda(), _i32(slots), k.view(E4M3), vt.view(E4M3), ke, ve)
        at, place = torch.tensor(slots, device="cuda") // page, torch.tensor(slots, device="cuda") % page
        assert torch.equal(k[at, :, place].cpu(), codes[:n]) and torch.equal(vt[at, :, :, place].cpu(), codes[:n])
        assert torch.equal(ke[at, :, place].cpu(), e[:n]) and torch.equal(ve[at, :, place].cpu(), e[:n])


# -------------------------------------------------------------------------------------- as they are used, one after the other
def test_a_prefill_over_a_quantised_cache_and_the_steps_after_it(spa):
    """Two prompts with the same first part: their keys are quantised, read back for the prefill of a next chunk with every block selected, then
    single tokens attend to the cache, with what they share and without; all as dense attention over the values that the cache stands for."""
    g = torch.Generator().manual_seed(12)
    page, Hq, Hkv, D = 64, 8, 2, 128
    prompt, chunk, steps = 320, 192, 4
    total = prompt + chunk + steps
    randn = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16)  # noqa: E731
    q = [randn(Hq, total, D) for _ in range(2)]
    k, v = ([randn(Hkv, total, D) for _ in range(2)] for _ in range(2))
    k[1][:, :prompt], v[1][:, :prompt] = k[0][:, :prompt], v[0][:, :prompt]
    stand = lambda x: oracle.values_of(*oracle.quantise(x)).to(torch.bfloat16)  # noqa: E731
    kq, vq = [stand(x) for x in k], [stand(x) for x in v]
    C = -(-total // page)
    n_pages = 2 * C + 1
    pages = [torch.full(s, 127, dtype=torch.uint8, device="cuda").view(E4M3) for s in ((n_pages, Hkv, page, D), (n_pages, Hkv, D, page))]
    exps = [torch.zeros((n_pages, Hkv, page), dtype=torch.uint8, device="cuda") for _ in range(2)]
    free = torch.randperm(n_pages, generator=g).to(torch.int32).cuda()
    table = torch.full((2, C), -1, dtype=torch.int32, device="cuda")
    # the prompt once, its pages in both rows
    starts, kv_lens, slots, _, taken = spa.paged_plan(table[:1], _i32([0]), _i32([prompt]), free, _i32([0, n_pages]), prompt, page, n_pages)
    spa.paged_append_q8(k[0][:, :prompt].transpose(0, 1).cuda(), v[0][:, :prompt].transpose(0, 1).cuda(), slots, *pages, *exps)
    used = int(taken[0])
    table[1] = table[0]
    # a chunk of each: behind what is read back
    new = [chunk, chunk]
    starts, kv_lens, slots, _, taken = spa.paged_plan(table, _i32([prompt] * 2), _i32(new), free, _i32([used, n_pages]), 2 * chunk, page, n_pages)
    used += int(taken[0])
    rows = slice(prompt, prompt + chunk)
    packed = lambda x, r: torch.cat([y[:, r].transpose(0, 1) for y in x]).cuda()  # noqa: E731
    spa.paged_append_q8(packed(k, rows), packed(v, rows), slots, *pages, *exps)
    out = spa.paged_attn_q8(packed(q, rows), *pages, *exps, table, starts, kv_lens, max_new_tokens=chunk)
    n = prompt + chunk
    back_k, back_v = (torch.empty((2, Hkv, n, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for b in range(2):
        spa.paged_read(*pages, table[b:b + 1], _i32([0, n]), kv_lens[b:b + 1], n, *exps, k=back_k[b].transpose(0, 1), v=back_v[b].transpose(0, 1))
        assert torch.equal(back_k[b].cpu(), kq[b][:, :n]) and torch.equal(back_v[b].cpu(), vq[b][:, :n])
    fused = spa.fused(torch.stack([x[:, rows] for x in q]).cuda(), back_k, back_v, 64, 1, 1, 4096)
    for b in range(2):
        want, _, tol, _ = paged_oracle.attn(q[b][:, rows].transpose(0, 1), [kq[b][:, :n]], [vq[b][:, :n]], [0, chunk], [n])
        assert ((out[b * chunk:(b + 1) * chunk].cpu().double() - want).abs() - tol).max().item() <= 0
        assert ((fused[b].transpose(0, 1).cpu().double() - want).abs() - tol).max().item() <= 0
    # single tokens, the groups found in the tables
    for i in range(steps):
        at = n + i
        starts, kv_lens, slots, _, taken = spa.paged_plan(table, _i32([at] * 2), _i32([1, 1]), free, _i32([used, n_pages]), 2, page, n_pages)
        used += int(taken[0])
        one = slice(at, at + 1)
        spa.paged_append_q8(packed(k, one), packed(v, one), slots, *pages, *exps)
        shares = spa.paged_shares(table, starts, kv_lens, page, 64)
        assert shares.tolist() == [[0, 0], [2, 2], [prompt, prompt]]
        alone = spa.paged_attn_q8(packed(q, one), *pages, *exps, table, starts, kv_lens, max_new_tokens=1)
        together = spa.paged_attn_shared(packed(q, one), *pages, table, starts, kv_lens, shares, *exps, max_new_tokens=1)
        for b in range(2):
            want, _, tol, _ = paged_oracle.attn(q[b][:, one].transpose(0, 1), [kq[b][:, :at + 1]], [vq[b][:, :at + 1]], [0, 1], [at + 1])
            for got in (alone, together):
                assert ((got[b:b + 1].cpu().double() - want).abs() - tol).max().item() <= 0


def test_a_captured_step_replays_with_other_lengths(spa):
    """Groups, quantising append, both attentions and the read back in one graph; eager calls in between."""
    page, Hq, Hkv, D, B, C = 16, 8, 2, 64, 5, 40
    n_pages = B * C
    g = torch.Generator().manual_seed(3)
    table = torch.randperm(n_pages, generator=g).view(B, C).to(torch.int32).cuda()
    pages = [torch.randint(0, 120, s, generator=g).to(torch.uint8).cuda().view(E4M3) for s in ((n_pages, Hkv, page, D), (n_pages, Hkv, D, page))]
    exps = [torch.randint(117, 124, (n_pages, Hkv, page), generator=g).to(torch.uint8).cuda() for _ in range(2)]
    starts, kv, slots, T, R = _i32([0] * (B + 1)), _i32([0] * B), _i32([-1] * 40), 40, 700
    q, k, v = (torch.randn((T, h, D), generator=g).to(torch.bfloat16).cuda() for h in (Hq, Hkv, Hkv))

    def step():
        spa.paged_append_q8(k, v, slots, *pages, *exps)
        shares = spa.paged_shares(table, starts, kv, page, 16)
        a = spa.paged_attn_q8(q, *pages, *exps, table, starts, kv, return_lse=True)
        b = spa.paged_attn_shared(q, *pages, table, starts, kv, shares, *exps, return_lse=True)
        rows = spa.paged_read(*pages, table, starts, kv, R, *exps)
        return (*a, *b, *rows, shares)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for turn, (lens, new, same) in enumerate([([16, 0, 300, 64, 9], [1, 0, 1, 1, 1], 3), ([640, 50, 30, 7, 632], [1, 30, 0, 7, 2], 0), ([10, 20, 30, 40, 50], [0, 0, 0, 0, 0], 9),
                                              ([600, 629, 512, 403, 640], [1, 9, 12, 3, 1], 20), ([200, 200, 200, 200, 200], [1, 1, 1, 1, 1], 12)]):
        table.copy_(torch.randperm(n_pages, generator=g).view(B, C).to(torch.int32).cuda())
        table[1:4, :same] = table[0, :same]
        kv.copy_(_i32(lens))
        starts.copy_(_i32([sum(new[:b]) for b in range(B + 1)]))
        places = [int(table[b, (lens[b] - new[b] + i) // page]) * page + (lens[b] - new[b] + i) % page for b in range(B) for i in range(new[b])]
        slots.copy_(_i32(places + [-1] * (T - len(places))))
        q.copy_(torch.randn(q.shape, generator=g).to(torch.bfloat16))
        graph.replay()
        again = step()
        torch.cuda.synchronize()
        end = sum(new)
        assert torch.equal(got[6], again[6])
        for x, y in zip(got[:6], again[:6]):
            assert torch.equal(x[:end], y[:end]), turn
        assert torch.isfinite(got[0][:end]).all()


def test_calls_on_two_streams_do_not_meet(spa):
    step = oracle.Step(11, [(1000, [(300, 1), (20, 60), (0, 1)]), (300, [(7, 1), (9, 1)])], q_heads=8, kv_heads=2, head_dim=64, q8=True)
    t = step.q.cuda(), *step.cache(), step.table.cuda(), _i32(step.starts), _i32(step.kv_lens), step.shares.cuda()
    calls = [lambda: spa.paged_attn_q8(*t[:-1]), lambda: spa.paged_attn_shared(t[0], t[1], t[2], *t[5:], t[3], t[4])]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for turn in range(8):
        with torch.cuda.stream(streams[turn // 2 % 2]):
            got.append((turn % 2, calls[turn % 2]()))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[i]) for i, x in got)


def test_more_requests_than_a_workgroup_has_threads(spa):
    """2000 requests, 4000 shares: several to a thread."""
    groups = [(80 + 16 * (x % 3), [((5 * b + x) % 60, (b + x) % 3) for b in range(1 + x % 5)]) for x in range(667)]
    step = oracle.Step(2000, groups, q_heads=2, kv_heads=1, head_dim=64, page=16, q8=True)
    assert len(step.kv_lens) > 1900
    out, lse = _attn(spa, step, shares=step.shares, return_lse=True)
    want, want_lse, tol, _ = step.want()
    assert ((out.cpu().double() - want).abs() - tol).max().item() <= 0
    found = spa.paged_shares(step.table.cuda(), _i32(step.starts), _i32(step.kv_lens), 16, 16)
    assert torch.equal(found.cpu(), oracle.shares(step.table, step.starts, step.kv_lens, 16, 16))


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_shared_attention_of_strided_tensors_and_one_workspace_for_many_calls(spa, q8):
    step = oracle.Step(3, [(300, [(20, 1), (0, 9)]), (70, [(5, 40), (1, 1), (0, 1)])], q_heads=6, kv_heads=2, page=64, q8=q8)
    T, B, N, C = step.T, 5, step.k_pages.shape[0], step.table.shape[1]
    kp, vp, ke, ve = step.cache()
    lens = _i32(step.starts), _i32(step.kv_lens)
    plain, lse = spa.paged_attn_shared(step.q.cuda(), kp, vp, step.table.cuda(), *lens, step.shares.cuda(), ke, ve, return_lse=True)
    qkv = torch.full((T, 10, 144), math.nan, dtype=torch.bfloat16, device="cuda")
    qkv[:, 2:8, 8:136] = step.q.cuda()
    both = torch.stack([kp.flatten(2).view(torch.uint8 if q8 else torch.bfloat16), vp.flatten(2).view(torch.uint8 if q8 else torch.bfloat16)], 1)
    k, v = both[:, 0].view(N, 2, 64, 128), both[:, 1].view(N, 2, 128, 64)
    if q8:
        k, v = k.view(E4M3), v.view(E4M3)
        both_exps = torch.stack([ke, ve], 2)
        ke, ve = both_exps[:, :, 0], both_exps[:, :, 1]
    wide = torch.full((B, 50), -1, dtype=torch.int32, device="cuda")
    wide[:, 3:3 + C] = step.table.cuda()
    room = torch.full((6, T, 160), 7.0, dtype=torch.bfloat16, device="cuda")
    need = spa.paged_shared_workspace_bytes(spa.make_paged_params(batch=B, n_q_heads=6, n_kv_heads=2, head_dim=128, page_size=64, n_pages=N, max_pages=C, n_tokens=T,
                                                                  table_stride=50))
    workspace = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    for turn in range(3):
        got, again = spa.paged_attn_shared(qkv[:, 2:8, 8:136], k, v, wide[:, 3:3 + C], *lens, step.shares.cuda(), ke, ve, out=room[:, :, 16:144].transpose(0, 1),
                                           workspace=workspace, return_lse=True)
        assert torch.equal(got.view(torch.int16), plain.view(torch.int16)) and torch.equal(again, lse), turn
        assert (room[:, :, :16] == 7.0).all() and (room[:, :, 144:] == 7.0).all()
        room.fill_(7.0)
        spa.paged_attn_shared(step.q.cuda()[:14], kp, vp, step.table.cuda()[:2], _i32([0, 1, 10]), lens[1][:2], step.shares[:, :2].cuda().contiguous(),
                              *step.cache()[2:], workspace=workspace)
    rows_k, rows_v = spa.paged_read(k, v, wide[:, 3:3 + C], _i32([0, 3, 3, 40, 41, 41]), lens[1], 41, ke, ve)
    assert torch.equal(rows_k[3:40].cpu(), step.keys[2][:, -37:].transpose(0, 1)) and torch.equal(rows_v[:3].cpu(), step.values[0][:, -3:].transpose(0, 1))


@pytest.mark.parametrize("n", [1, 31, 1024, 1025])
def test_append_of_either_kernel_leaves_the_same_bytes(spa, n):
    """A prompt that starts inside a page, in one call and token by token (33 at a time)."""
    page, H, D = 32, 3, 64
    x = torch.randn(2, n, H, D, generator=torch.Generator().manual_seed(n)).to(torch.bfloat16).cuda()
    slots = torch.arange(5, 5 + n, dtype=torch.int32, device="cuda")
    caches = []
    for size in (n, 33):
        c = [torch.full(s, 9, dtype=torch.uint8, device="cuda") for s in ((40, H, page, D), (40, H, D, page), (40, H, page), (40, H, page))]
        for at in range(0, n, size):
            part = slice(at, at + size)
            spa.paged_append_q8(x[0, part], x[1, part], slots[part].contiguous(), c[0].view(E4M3), c[1].view(E4M3), *c[2:])
        caches.append(c)
    assert all(torch.equal(a, b) for a, b in zip(*caches))


def test_nothing_to_do(spa):
    """No tokens at all, one request, the shortest lengths."""
    step = oracle.Step(1, [(64, [(0, 1), (0, 1)])], q8=True, padding=5)
    kp, vp, ke, ve = step.cache()
    out = torch.full((step.T, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    zero = _i32([0, 0, 0])
    spa.paged_attn_shared(step.q.cuda(), kp, vp, step.table.cuda(), zero, _i32(step.kv_lens), step.shares.cuda(), ke, ve, out=out)
    spa.paged_attn_q8(step.q.cuda(), kp, vp, ke, ve, step.table.cuda(), zero, _i32(step.kv_lens), out=out)
    assert (out == 7.0).all()
    k = torch.full((3, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    v = k.clone()
    spa.paged_read(kp, vp, step.table.cuda(), zero, _i32(step.kv_lens), 3, ke, ve, k=k, v=v)
    assert (k == 7.0).all() and (v == 7.0).all()
    before = kp.view(torch.uint8).clone()
    spa.paged_append_q8(k, v, _i32([-1, -1, 2 ** 31 - 1]), kp, vp, ke, ve)
    assert torch.equal(kp.view(torch.uint8), before)
    assert spa.paged_shares(step.table[:1].cuda(), _i32([0, 1]), _i32([65]), 64, 0).tolist() == [[0], [1], [0]]
