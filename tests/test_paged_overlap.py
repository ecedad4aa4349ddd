"""Paged calls refuse arrays that lie on each other: the rule (csrc/overlap.hpp, compiled for the host) against every byte, and the calls."""
import ctypes
import random

import pytest

from host_shim import compile_shim
from test_paged_abi import FAKE, _append, _attn, _params, lib  # noqa: F401  (a fixture)

SOURCE = '''
#include "overlap.hpp"
using namespace spa;
static Rows rows(const long long* x) { return rows_of((const void*)x[0], x[1], x[2], x[3], x[4], x[5]); }
extern "C" int meet(const long long* a, const long long* b) { return overlap(rows(a), rows(b)); }
extern "C" int self(const long long* a) { return overlaps_itself(rows(a)); }
'''


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    return compile_shim(tmp_path_factory.mktemp("overlap"), SOURCE)


def _c(x):
    return (ctypes.c_longlong * 6)(*x)


def _bytes(x):
    at, n0, s0, n1, s1, n = x
    return [at + i * s0 + j * s1 + b for i in range(n0) for j in range(n1) for b in range(n)]


def _draw(r, strides=None):
    s0, s1 = strides or (r.choice((0, 3, 8, 17, 40)), r.choice((0, 2, 5, 8, 30)))
    return 1000 + r.randint(0, 120), r.randint(1, 4), s0, r.randint(1, 4), s1, r.randint(1, 9)


def test_rows_of_the_same_strides_meet_where_a_byte_is_in_both(shim):
    r = random.Random(1)
    seen = set()
    for _ in range(6000):
        a = _draw(r)
        b = _draw(r, (a[2], a[4]))
        want = not set(_bytes(a)).isdisjoint(_bytes(b))
        assert bool(shim.meet(_c(a), _c(b))) == want and bool(shim.meet(_c(b), _c(a))) == want, (a, b)
        seen.add(want)
    assert seen == {False, True}


def test_a_single_row_meets_rows_where_a_byte_is_in_both_and_no_meeting_is_missed(shim):
    r = random.Random(2)
    for _ in range(6000):
        a, b = _draw(r), _draw(r)
        single = (b[0], 1, b[2], 1, b[4], b[5])
        want = not set(_bytes(a)).isdisjoint(_bytes(single))
        assert bool(shim.meet(_c(a), _c(single))) == want and bool(shim.meet(_c(single), _c(a))) == want
        if not set(_bytes(a)).isdisjoint(_bytes(b)):
            assert shim.meet(_c(a), _c(b))
        if max(_bytes(a)) < min(_bytes(b)):
            assert not shim.meet(_c(a), _c(b))


def test_rows_that_lie_on_each_other_are_found(shim):
    r = random.Random(3)
    for _ in range(6000):
        a = _draw(r)
        assert bool(shim.self(_c(a))) == (len(set(_bytes(a))) < len(_bytes(a))), a
    assert not shim.self(_c((1000, 1, 0, 1, 0, 8)))


def test_strides_of_any_size_do_not_wrap(shim):
    far = (1000, 3, 2 ** 62, 2, 2 ** 61, 8)
    assert not shim.self(_c(far)) and shim.meet(_c(far), _c((1000 + 2 ** 62, 1, 0, 1, 0, 1))) and not shim.meet(_c(far), _c((1008 + 2 ** 62, 1, 0, 1, 0, 1)))
    assert not shim.meet(_c((0, 1, 0, 1, 0, 8)), _c((0, 1, 0, 1, 0, 8)))       # no array


# The arrays of a call, far apart; what each takes in bytes (30 tokens, 8 and 2 heads of 128, 100 pages of 64)
ATTN = ("q", "k", "vt", "table", "starts", "kv", "slopes", "out", "lse")
PLACE = {n: FAKE + (i + 1) * 0x10000000 for i, n in enumerate(ATTN)}
SIZE = dict(q=30 * 2048, k=100 * 32768, vt=100 * 32768, table=240, starts=16, kv=12, slopes=32, out=30 * 2048, lse=30 * 32)


def test_attention_refuses_outputs_on_other_arrays(lib):  # noqa: F811
    p = _params()
    for written in ("out", "lse"):
        for other in ATTN:
            if other == written:
                continue
            for at in (PLACE[other], PLACE[other] + SIZE[other] - 16 if SIZE[other] > 16 else PLACE[other], PLACE[other] - SIZE[written] + 16):
                at = at // 16 * 16
                assert _attn(lib, p, dict(PLACE, **{written: at}), ws=FAKE) == -8, (written, other)


def test_attention_refuses_a_workspace_on_other_arrays(lib):  # noqa: F811
    p = _params(max_pages=2000, table_stride=2000)
    for other in ATTN:
        assert _attn(lib, p, PLACE, ws=PLACE[other]) == -8, other


def test_attention_refuses_an_output_inside_the_packed_queries(lib):  # noqa: F811
    """q and out as slices of one tensor [tokens, 25 heads]: one head too near, rows of another token."""
    p = _params(q=(3200, 128), out=(3200, 128))
    for shift in (7 * 128, -7 * 128, 3200 - 7 * 128, 8):
        assert _attn(lib, p, dict(PLACE, out=PLACE["q"] + 0x4000 + 2 * shift, q=PLACE["q"] + 0x4000), ws=FAKE) == -8
    assert _attn(lib, _params(q=(2048, 128), out=(1024, 128)), dict(PLACE, out=PLACE["q"] + 2048), ws=FAKE) == -8


@pytest.mark.parametrize("out", [(128, 128), (256, 128), (128, 256), (136, 128)])
def test_attention_refuses_an_output_on_itself(lib, out):  # noqa: F811
    assert _attn(lib, _params(out=out), PLACE, ws=FAKE) == -8


def test_append_refuses_pages_on_each_other_and_inputs_in_the_cache(lib):  # noqa: F811
    place = dict(k=FAKE, v=FAKE + 0x1000000, slots=FAKE + 0x2000000, k_pages=FAKE + 0x10000000, vt_pages=FAKE + 0x20000000)
    p = _params()
    assert _append(lib, p, dict(place, vt_pages=place["k_pages"] + 100 * 32768 - 16)) == -8
    both = _params(k_pages=(32768, 8192), vt_pages=(32768, 8192))         # one allocation, K and V a page of two heads apart
    assert _append(lib, both, dict(place, vt_pages=place["k_pages"] + 16384)) == -8
    for name in ("k", "v", "slots"):
        assert _append(lib, p, {**place, name: place["vt_pages"] + 99 * 32768}) == -8, name
    assert _append(lib, _params(k_pages=(8192, 8192)), place) == -8
