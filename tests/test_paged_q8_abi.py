"""Host-side checks of the quantised cache's calls and of those for shared prompts, without a GPU: bad arguments are refused before any launch."""
import ctypes

import pytest
import torch

import paper_2602_21233_amd as spa
from paper_2602_21233_amd import binding
from test_paged_abi import _params as _bf16_params
from test_paged_abi import lib  # noqa: F401  (a fixture)

AT = {n: 0x100000 + 0x10000000 * (i + 1) for i, n in enumerate(                   # never dereferenced on the host
    ("q", "k", "v", "slots", "k_pages", "vt_pages", "k_exp", "v_exp", "table", "starts", "kv", "shares", "slopes", "out", "lse", "ws"))}


def _params(**kw):
    return _bf16_params(**{**dict(k_pages=(16384, 8192), vt_pages=(16384, 8192)), **kw})


def _exps(k=AT["k_exp"], v=AT["v_exp"], k_stride=(128, 64), v_stride=(128, 64)):
    return binding.SpaPagedExps(k, v, (ctypes.c_int64 * 2)(*k_stride), (ctypes.c_int64 * 2)(*v_stride))


def _append(lib, p, exps=None, **at):  # noqa: F811
    a = {**AT, **at}
    e = _exps() if exps is None else exps
    return lib.sparse_prefill_paged_append_quantised(ctypes.byref(p), a["k"], a["v"], a["slots"], a["k_pages"], a["vt_pages"], ctypes.byref(e) if e else None, None)


def _attn(lib, p, exps=None, ws_bytes=1 << 40, **at):  # noqa: F811
    a = {**AT, **dict(slopes=None, lse=None), **at}
    e = _exps() if exps is None else exps
    return lib.sparse_prefill_paged_attn_quantised(ctypes.byref(p), a["q"], a["k_pages"], a["vt_pages"], ctypes.byref(e) if e else None, a["table"], a["starts"],
                                                   a["kv"], a["slopes"], a["out"], a["lse"], a["ws"], ws_bytes, None)


def _shared(lib, p, exps=None, ws_bytes=1 << 40, **at):  # noqa: F811
    a = {**AT, **dict(slopes=None, lse=None), **at}
    e = _exps() if exps is None else exps
    return lib.sparse_prefill_paged_attn_shared(ctypes.byref(p), a["q"], a["k_pages"], a["vt_pages"], ctypes.byref(e) if e else None, a["table"], a["starts"],
                                                a["kv"], a["shares"], a["slopes"], a["out"], a["lse"], a["ws"], ws_bytes, None)


def _read(lib, p, exps=None, **at):  # noqa: F811
    a = {**AT, **at}
    e = _exps() if exps is None else exps
    return lib.sparse_prefill_paged_read(ctypes.byref(p), a["k_pages"], a["vt_pages"], ctypes.byref(e) if e else None, a["table"], a["starts"], a["kv"], a["k"],
                                         a["v"], None)


def _shares(lib, p, least=1, **at):  # noqa: F811
    a = {**AT, **at}
    return lib.sparse_prefill_paged_shares(ctypes.byref(p), a["table"], a["starts"], a["kv"], least, a["shares"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), -2), (dict(batch=4097), -2), (dict(n_q_heads=7), -2), (dict(n_kv_heads=0), -2), (dict(head_dim=96), -2), (dict(page_size=8), -2),
    (dict(n_pages=0), -2), (dict(max_pages=0), -2), (dict(n_tokens=0), -2), (dict(n_tokens=2 ** 24 + 1), -2), (dict(max_new_tokens=-1), -2),
    (dict(softmax_scale=float("nan")), -2), (dict(window_tokens=-1), -3), (dict(softcap=-1.0), -3), (dict(softcap=65537.0), -3)])
def test_bad_params_are_refused_by_every_call(lib, kw, code):  # noqa: F811
    p = _params(**kw)
    n = ctypes.c_size_t()
    assert lib.spa_paged_shared_workspace_bytes(ctypes.byref(p), ctypes.byref(n)) == code
    assert all(call(lib, p) == code for call in (_append, _attn, _shared, _read, _shares))


def test_null_and_misaligned_pointers_are_refused(lib):  # noqa: F811
    p, n = _params(), ctypes.c_size_t()
    assert lib.spa_paged_shared_workspace_bytes(None, ctypes.byref(n)) == -1 and lib.spa_paged_shared_workspace_bytes(ctypes.byref(p), None) == -1
    needed = {_append: ("k", "v", "slots", "k_pages", "vt_pages"), _attn: ("q", "k_pages", "vt_pages", "table", "starts", "kv", "out"),
              _shared: ("q", "k_pages", "vt_pages", "table", "starts", "kv", "shares", "out", "ws"), _read: ("k_pages", "vt_pages", "table", "starts", "kv", "k", "v"),
              _shares: ("table", "starts", "kv", "shares")}
    for call, names in needed.items():
        for name in names:
            assert call(lib, p, **{name: None}) == -1, (call.__name__, name)
            if name in ("q", "k", "v", "k_pages", "vt_pages", "out"):
                assert call(lib, p, **{name: AT[name] + 8}) == -4, (call.__name__, name)
    for call in (_append, _attn, _shared, _read):
        assert call(lib, p, exps=_exps(k=None)) == -1 and call(lib, p, exps=_exps(v=None)) == -1
        assert call(lib, p, exps=_exps(k=AT["k_exp"] + 8)) == -4
    assert _append(lib, p, exps=False) == -1 and _attn(lib, p, exps=False) == -1            # no exponents: not a quantised cache
    assert _shared(lib, p, ws=AT["ws"] + 16) == -4 and _shared(lib, p, ws_bytes=16) == -5
    assert _shares(lib, p, least=-1) == -3


@pytest.mark.parametrize("kw", [dict(k_pages=(16384, 8200)), dict(k_pages=(16392, 8192)), dict(vt_pages=(16384, 8200)), dict(vt_pages=(4096, 8192))])
def test_bad_page_strides_are_refused(lib, kw):  # noqa: F811
    p = _params(**kw)
    assert all(call(lib, p) == -4 for call in (_append, _attn, _shared, _read))


@pytest.mark.parametrize("kw", [dict(k_stride=(128, 72)), dict(v_stride=(136, 64)), dict(k_stride=(128, 48)), dict(v_stride=(-128, 64))])
def test_bad_strides_of_exponents_are_refused(lib, kw):  # noqa: F811
    p = _params()
    assert all(call(lib, p, exps=_exps(**kw)) == -4 for call in (_append, _attn, _shared, _read))


def test_other_bad_strides_are_refused(lib):  # noqa: F811
    assert _read(lib, _params(k=(256, 64))) == -4 and _read(lib, _params(v=(0, 128))) == -4 and _read(lib, _params(table_stride=19)) == -4
    assert _shared(lib, _params(out=(1024, 64))) == -4 and _shared(lib, _params(table_stride=19)) == -4 and _shares(lib, _params(table_stride=19)) == -4
    assert _attn(lib, _params(q=(1024, 129))) == -4 and _append(lib, _params(k=(256, 129))) == -4


SIZE = dict(q=30 * 2048, k=30 * 512, v=30 * 512, slots=120, k_pages=100 * 16384, vt_pages=100 * 16384, k_exp=12800, v_exp=12800, table=240, starts=16, kv=12,
            shares=36, slopes=32, out=30 * 2048, lse=30 * 32)


@pytest.mark.parametrize("call,written,others", [
    (_append, ("k_pages", "vt_pages", "k_exp", "v_exp"), ("k", "v", "slots", "k_pages", "vt_pages", "k_exp", "v_exp")),
    (_attn, ("out", "lse"), ("q", "k_pages", "vt_pages", "k_exp", "v_exp", "table", "starts", "kv", "slopes", "out", "lse")),
    (_shared, ("out", "lse", "ws"), ("q", "k_pages", "vt_pages", "k_exp", "v_exp", "table", "starts", "kv", "shares", "slopes", "out", "lse")),
    (_read, ("k", "v"), ("k_pages", "vt_pages", "k_exp", "v_exp", "table", "starts", "kv", "k", "v")),
    (_shares, ("shares",), ("table", "starts", "kv"))], ids=["append", "attn", "shared", "read", "shares"])
def test_arrays_on_each_other_are_refused(lib, call, written, others):  # noqa: F811
    p = _params()
    for name in written:
        for other in others:
            if other == name:
                continue
            for at in {AT[other], AT[other] + max(0, SIZE[other] - 16) // 256 * 256}:
                place = dict(AT, **{name: at})
                kw = dict(place) if call not in (_append, _attn, _shared, _read) else dict(place, exps=_exps(k=place["k_exp"], v=place["v_exp"]))
                assert call(lib, p, **kw) == -8, (name, other)


def test_one_tensor_for_keys_and_values_is_refused(lib):  # noqa: F811
    p = _params()
    for call in (_attn, _shared, _read):
        assert call(lib, p, vt_pages=AT["k_pages"]) == -8 and call(lib, p, exps=_exps(v=AT["k_exp"])) == -8


def test_workspace_of_shared_prompts(lib):  # noqa: F811
    def need(**kw):
        return spa.paged_shared_workspace_bytes(_params(**kw))
    assert need() % 256 == 0 and need(max_pages=2000) >= need()
    assert need(max_pages=2000, batch=64, n_tokens=64) <= 256 << 20
    assert need(max_pages=2000, batch=4096, n_tokens=4096) <= 2 << 30
    # two results of every row in 32 bits, and what the cuts add
    assert need(max_pages=2000, batch=4, n_tokens=8192, n_q_heads=32, n_kv_heads=8) <= 2 * 8192 * 32 * 129 * 4 + (512 << 20)


def test_binding_refuses_other_types_and_shapes():
    t = torch.zeros(4, dtype=torch.int32)
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    pages, vt = torch.zeros((3, 2, 16, 64), dtype=torch.float8_e4m3fn), torch.zeros((3, 2, 64, 16), dtype=torch.float8_e4m3fn)
    exps = torch.zeros((3, 2, 16), dtype=torch.uint8)
    for bad in (lambda: spa.paged_append_q8(x, x, t, pages, vt, exps, exps), lambda: spa.paged_attn_q8(x, pages, vt, exps, exps, t.view(2, 2), t[:3], t[:2]),
                lambda: spa.paged_read(pages, vt, t.view(2, 2), t[:3], t[:2], 4, exps, exps), lambda: spa.paged_shares(t.view(2, 2), t[:3], t[:2], 16),
                lambda: spa.paged_attn_shared(x, pages, vt, t.view(2, 2), t[:3], t[:2], torch.zeros((3, 2), dtype=torch.int32), exps, exps)):
        with pytest.raises(TypeError):
            bad()


def test_packed_exponents_equal_their_fields():
    from paper_2602_21233_amd import paged
    e = binding.SpaPagedExps.from_buffer_copy(paged._EXPS.pack(1, 2, 3, 4, 5, 6))
    assert (e.k, e.v, tuple(e.k_stride), tuple(e.v_stride)) == (1, 2, (3, 4), (5, 6))
