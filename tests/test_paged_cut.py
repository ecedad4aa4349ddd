"""How an attention call over pages is cut (csrc/paged.hpp, compiled for the host), against every row's own keys."""
import ctypes

import pytest

from host_shim import compile_shim

SOURCE = '''
#include "paged.hpp"
using namespace spa;
extern "C" void tiles_of(int lo, int hi, int sink, int window, int* out) { const KeyTiles t = key_tiles(lo, hi, sink, window); out[0] = t.sinks; out[1] = t.from; out[2] = t.n; }
extern "C" int most(int q_len, int kv, int span, int sink, int window) { return most_key_tiles(q_len, kv, span, sink, window); }
extern "C" int piece(long long work, int log_most, int min_tiles, int few) { PagedPart p{}; p.log_most = log_most; p.min_tiles = min_tiles; return few ? few_rows_piece(work, p) : shortest_piece(work, p); }
extern "C" void share(int m, int log_m, int span, int G, int q_len, int kv, int sink, int window, int piece, int* out) {
    PagedPart p{}; p.m = m; p.log_m = log_m; p.span = span; p.row_lo = 0; p.row_hi = 0x7fffffff;
    const PagedShare s = paged_share(p, G, q_len, kv, sink, window, piece); out[0] = s.tiles; out[1] = s.keys; out[2] = s.splits; }
'''


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    return compile_shim(tmp_path_factory.mktemp("cut"), SOURCE)


@pytest.mark.parametrize("sink", [0, 1, 63, 64, 65, 300, 2 ** 30])
@pytest.mark.parametrize("window", [0, 1, 2, 64, 100, 500, 2 ** 30])
@pytest.mark.parametrize("m,G", [(16, 1), (16, 4), (16, 5), (16, 40), (32, 3), (128, 1), (128, 4), (128, 5), (128, 70)])
def test_every_seen_key_lies_in_a_tile_and_tiles_ascend(shim, sink, window, m, G):
    span = (m + G - 1) // G + 1
    out = (ctypes.c_int * 3)()
    for q_len, kv in ((1, 1), (1, 64), (1, 700), (1, 1025), (9, 5), (9, 9), (70, 640), (200, 200), (130, 1000), (3, 0)):
        rows, keys = q_len * G, shim.most(q_len, kv, span, sink, window)
        longest = 0
        for r0 in range(0, rows, m):
            lo, hi = kv - q_len + r0 // G, kv - q_len + (min(r0 + m, rows) - 1) // G
            assert hi - lo + 1 <= span
            shim.tiles_of(lo, hi, sink, window, out)
            sinks, start, n = out
            tiles = [e if e < sinks else e - sinks + start for e in range(n)]
            assert tiles == sorted(set(tiles)) and (not tiles or tiles[-1] == hi // 64)
            seen = {j // 64 for i in {max(lo, 0), hi} if 0 <= i <= hi for j in range(i + 1) if not window or i - j < window or j < sink}
            assert seen <= set(tiles), (q_len, kv, r0)
            longest = max(longest, n)
        assert longest <= keys <= max(longest + 3, (kv + 63) // 64 if not window else longest + 3)


@pytest.mark.parametrize("log_most,min_tiles,few", [(10, 2, 0), (11, 4, 1)])
def test_pieces_stay_in_the_workspace(shim, log_most, min_tiles, few):
    out = (ctypes.c_int * 3)()
    for Hkv in (1, 8):
        for lens in ([131072], [131072, 90000, 1, 3], [100] * 60 + [50000], [8191] * 64, [10] * 4096, [2 ** 30]):
            work = 0
            for kv in lens:
                shim.share(16, 4, 5, 4, 1, kv, 0, 0, 2 ** 24, out)
                assert list(out) == [1, (kv + 63) // 64, 1]
                work += out[0] * out[1] * Hkv
            piece = shim.piece(ctypes.c_longlong(work), log_most, min_tiles, few)
            assert piece >= min_tiles
            assert not few or piece <= max(16, -(-work // 2 ** log_most))
            units = slots = 0
            for kv in lens:
                shim.share(16, 4, 5, 4, 1, kv, 0, 0, piece, out)
                assert out[2] * piece >= out[1] and (out[2] == 1 or out[1] > piece)
                per = -(-out[1] // out[2])
                assert per * out[2] >= out[1] and per <= piece
                units += out[0] * out[2] * Hkv
                slots += out[0] * out[2] * Hkv if out[2] > 1 else 0
            assert units <= 2 ** log_most + len(lens) * Hkv and slots <= 2 * 2 ** log_most


@pytest.mark.parametrize("sink,window", [(0, 0), (0, 1), (5, 64), (64, 100), (300, 500), (0, 4096), (2 ** 30, 2 ** 30)])
@pytest.mark.parametrize("m,G", [(16, 4), (32, 3), (128, 1), (128, 5), (128, 70)])
def test_no_request_has_more_key_tiles_than_the_table_allows(shim, sink, window, m, G):
    """What the host lays out from the table's width and all the tokens holds for each request's own lengths."""
    span = (m + G - 1) // G + 1
    for total, width in ((1, 64), (7, 16), (200, 1000), (4096, 8192), (2 ** 24, 2 ** 30)):
        most = shim.most(total, width, span, sink, window)
        for q_len in {1, 2, total // 2 or 1, total}:
            for kv in {0, 1, 63, 64, width // 2, width - 1, width}:
                if q_len <= total and kv <= width:
                    assert shim.most(q_len, kv, span, sink, window) <= most
