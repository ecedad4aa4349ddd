"""Host-side checks of the paged-KV-cache calls, without a GPU: bad arguments are refused before any launch."""
import ctypes

import pytest
import torch

import paper_2602_21233_amd as spa
from paper_2602_21233_amd import binding

FAKE = 0x100000                      # never dereferenced on the host


@pytest.fixture(scope="module")
def lib():
    return spa.load_library()


def _params(**kw):
    base = dict(batch=3, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=64, n_pages=100, max_pages=20, n_tokens=30, table_stride=20,
                q=(1024, 128), k=(256, 128), v=(256, 128), out=(1024, 128), k_pages=(16384, 8192), vt_pages=(16384, 8192))
    base.update(kw)
    return spa.make_paged_params(**base)


def _attn(lib, p, change=None, ws=FAKE, ws_bytes=1 << 40):
    a = dict(q=FAKE, k=FAKE, vt=FAKE, table=FAKE, starts=FAKE, kv=FAKE, slopes=None, out=FAKE, lse=None)
    a.update(change or {})
    return lib.sparse_prefill_paged_attn(ctypes.byref(p), *a.values(), ws, ws_bytes, None)


def _append(lib, p, change=None):
    a = dict(k=FAKE, v=FAKE, slots=FAKE, k_pages=FAKE, vt_pages=FAKE)
    a.update(change or {})
    return lib.sparse_prefill_paged_append(ctypes.byref(p), *a.values(), None)


PLAN = ("ctx", "new", "free", "range", "table", "starts", "kv", "slots", "positions", "taken")


def _plan(lib, p, change=None, n_free=50):
    a = {n: FAKE + 0x10000 * i for i, n in enumerate(PLAN)}
    a.update(change or {})
    args = list(a.values())
    return lib.sparse_prefill_paged_plan(ctypes.byref(p), *args[:3], n_free, *args[3:], None)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), -2), (dict(batch=4097), -2), (dict(n_q_heads=7), -2), (dict(n_kv_heads=0), -2), (dict(n_q_heads=0), -2),
    (dict(head_dim=96), -2), (dict(head_dim=256), -2), (dict(page_size=8), -2), (dict(page_size=48), -2), (dict(page_size=256), -2),
    (dict(n_pages=0), -2), (dict(n_pages=2 ** 25, page_size=64), -2), (dict(max_pages=0), -2), (dict(max_pages=2 ** 24 + 1), -2),
    (dict(n_tokens=0), -2), (dict(n_tokens=2 ** 24 + 1), -2), (dict(n_tokens=2 ** 24, n_q_heads=256, n_kv_heads=2), -2), (dict(max_new_tokens=-1), -2),
    (dict(softmax_scale=-1.0), -2), (dict(softmax_scale=float("nan")), -2), (dict(softmax_scale=float("inf")), -2),
    (dict(n_sink_tokens=-1), -3), (dict(window_tokens=-1), -3), (dict(softcap=-1.0), -3), (dict(softcap=float("nan")), -3), (dict(softcap=float("inf")), -3), (dict(softcap=65537.0), -3),
])
def test_bad_params_are_refused_by_every_call(lib, kw, code):
    p = _params(**kw)
    n = ctypes.c_size_t()
    assert lib.spa_paged_workspace_bytes(ctypes.byref(p), ctypes.byref(n)) == code
    assert _plan(lib, p) == code and _append(lib, p) == code and _attn(lib, p) == code


def test_null_and_misaligned_pointers_are_refused(lib):
    p = _params()
    n = ctypes.c_size_t()
    assert lib.spa_paged_workspace_bytes(None, ctypes.byref(n)) == -1 and lib.spa_paged_workspace_bytes(ctypes.byref(p), None) == -1
    for name in PLAN:
        if name != "positions":
            assert _plan(lib, p, {name: None}) == -1, name
    assert _plan(lib, p, n_free=-1) == -2
    for name in ("k", "v", "slots", "k_pages", "vt_pages"):
        assert _append(lib, p, {name: None}) == -1, name
        if name != "slots":
            assert _append(lib, p, {name: FAKE + 8}) == -4, name
    for name in ("q", "k", "vt", "table", "starts", "kv", "out"):
        assert _attn(lib, p, {name: None}) == -1, name
        if name in ("q", "k", "vt", "out"):
            assert _attn(lib, p, {name: FAKE + 8}) == -4, name
    assert _attn(lib, p, ws=None) == -1 and _attn(lib, p, ws=FAKE + 16) == -4 and _attn(lib, p, ws_bytes=16) == -5


@pytest.mark.parametrize("kw", [dict(table_stride=19), dict(q=(1024, 129)), dict(q=(-1024, 128)), dict(out=(1024, 64)), dict(out=(0, 128)),
                                dict(k_pages=(16384, 4096)), dict(k_pages=(8184, 8192)), dict(vt_pages=(16385, 8192)), dict(vt_pages=(16384, 0))])
def test_bad_strides_are_refused_by_attn(lib, kw):
    assert _attn(lib, _params(**kw)) == -4


@pytest.mark.parametrize("kw", [dict(k=(256, 129)), dict(v=(-256, 128)), dict(k_pages=(16384, 4096)), dict(vt_pages=(16385, 8192))])
def test_bad_strides_are_refused_by_append(lib, kw):
    assert _append(lib, _params(**kw)) == -4


def test_plan_refuses_arrays_that_overlap(lib):
    p, size = _params(), dict(ctx=3, new=3, free=50, range=2, table=60, starts=4, kv=3, slots=30, positions=30, taken=2)
    for i, out in enumerate(PLAN):
        if i < 4:
            continue
        for other in PLAN:
            if other != out:
                at = FAKE + 0x10000 * PLAN.index(other)
                assert _plan(lib, p, {out: at + 4 * (size[other] - 1)}) == -8, (out, other)
    assert "overlap" in lib.spa_strerror(-8).decode()


def test_workspace_covers_the_cut_rows_and_no_more_than_it_must(lib):
    def need(**kw):
        return spa.paged_workspace_bytes(_params(**kw))
    assert need(max_pages=1) == 0                                    # nothing to cut
    assert need(max_pages=2000) > 0
    assert need(max_pages=2000, batch=4096, n_tokens=2 ** 14) <= 256 << 20
    assert need(max_pages=2000) % 256 == 0


def test_values_that_do_not_fit_a_field_are_refused():
    with pytest.raises(spa.SpaError):
        _params(n_tokens=2 ** 31)
    with pytest.raises(spa.SpaError):
        spa.paged_workspace_bytes(_params(softcap=1e300))      # infinite as a float


def test_binding_refuses_what_is_not_on_the_gpu():
    t = torch.zeros(4, dtype=torch.int32)
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    pages, vt = torch.zeros((3, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((3, 2, 64, 16), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        spa.paged_append(x, x, t, pages, vt)
    with pytest.raises(TypeError):
        spa.paged_attn(x, pages, vt, t.view(2, 2), t[:3], t[:2])
    with pytest.raises((TypeError, ValueError)):
        spa.paged_plan(t.view(2, 2), t[:2], t[:2], t, t[:2], 4, 16, 3)


def test_packed_params_equal_their_fields():
    p = _params(softmax_scale=0.25, n_sink_tokens=5, window_tokens=6, softcap=7.5, max_new_tokens=4)
    assert [getattr(p, n) for n, _ in binding.SpaPagedParams._fields_[:14]] == [3, 8, 2, 128, 64, 100, 20, 30, 4, 0.25, 5, 6, 7.5, 20]
    assert [tuple(getattr(p, n)) for n, _ in binding.SpaPagedParams._fields_[14:]] == [(1024, 128), (256, 128), (256, 128), (1024, 128), (16384, 8192), (16384, 8192)]


def test_attention_in_place_and_one_tensor_for_k_and_v_pages_are_refused(lib):
    p = _params()
    assert _attn(lib, p, dict(out=FAKE, q=FAKE, k=FAKE + 0x1000, vt=FAKE + 0x2000)) == -8
    assert _attn(lib, p, dict(out=FAKE + 0x1000, q=FAKE, k=FAKE + 0x2000, vt=FAKE + 0x2000)) == -8
    assert _append(lib, p, dict(k_pages=FAKE + 0x1000, vt_pages=FAKE + 0x1000)) == -8
