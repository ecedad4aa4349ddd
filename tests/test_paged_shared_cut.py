"""How a call with shared prompts is cut (csrc/paged.hpp, compiled for the host), against every row's own keys; and what the kernels take of a SIMD."""
import ctypes

import pytest

from host_shim import compile_shim
from test_kernel_resources import kernels  # noqa: F401  (a fixture)

SOURCE = '''
#include "paged.hpp"
using namespace spa;
extern "C" void tiles_of(int lo, int hi, int sink, int window, int first, int end, int* out) {
    const KeyTilesWithin t = key_tiles_within(lo, hi, sink, window, first, end); out[0] = t.n; for (int e = 0; e < t.n; ++e) out[1 + e] = t.at(e); }
extern "C" void all_of(int lo, int hi, int sink, int window, int* out) {
    const KeyTiles t = key_tiles(lo, hi, sink, window); out[0] = t.n; for (int e = 0; e < t.n; ++e) out[1 + e] = t.at(e); }
extern "C" void share(int m, int log_m, int lo, int hi, int span, int G, int len, int tile, int end, int kv, int members, int sink, int window, int* out) {
    PagedPart p{}; p.m = m; p.log_m = log_m; p.span = span; p.row_lo = lo; p.row_hi = hi;
    const SharedInfo r{0, len, tile, end, kv, members, 0, 0};
    const PagedShare s = shared_share(p, G, r, sink, window); out[0] = s.tiles; out[1] = s.keys; }
'''


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    return compile_shim(tmp_path_factory.mktemp("shared_cut"), SOURCE)


@pytest.mark.parametrize("sink", [0, 1, 64, 65, 300, 2 ** 30])
@pytest.mark.parametrize("window", [0, 1, 64, 100, 700, 2 ** 30])
def test_common_and_own_tiles_are_all_tiles_once(shim, sink, window):
    out = (ctypes.c_int * 100)()

    def ask(f, *a):
        f(*a, out)
        return list(out[1:1 + out[0]])

    for lo, hi in ((0, 0), (63, 63), (64, 70), (500, 640), (1000, 1000), (-5, 3), (-9, -1), (2000, 2130)):
        want = ask(shim.all_of, lo, hi, sink, window)
        for cut in (0, 1, 3, 10, 16, 40):
            common, own = ask(shim.tiles_of, lo, hi, sink, window, 0, cut), ask(shim.tiles_of, lo, hi, sink, window, cut, 1 << 24)
            assert common + own == want, (lo, hi, cut)
            assert all(t < cut for t in common) and all(t >= cut for t in own)


@pytest.mark.parametrize("m,log_m,row_lo,row_hi", [(16, 4, 0, 16), (32, 5, 0, 32), (128, 7, 16, 2 ** 31 - 1)])
def test_a_share_has_room_for_every_row_tile(shim, m, log_m, row_lo, row_hi):
    out = (ctypes.c_int * 100)()
    for G in (1, 4, 5, 16, 40):
        span = (m + G - 1) // G + 1
        for length in (0, 1, 3, 4, 60, 700):
            for kv, cut in ((0, 0), (length, 0), (1000, 3), (1000, 15), (1000, 40), (700, 2)):
                for sink, window in ((0, 0), (70, 100), (0, 1), (2000, 5)):
                    shim.share(m, log_m, row_lo, row_hi, span, G, length, cut, 1 << 24, kv, 0, sink, window, out)
                    tiles, keys = out[0], out[1]
                    rows = length * G
                    assert tiles == (-(-rows // m) if row_lo < rows <= row_hi else 0)
                    for r0 in range(0, rows if tiles else 0, m):
                        lo, hi = kv - length + r0 // G, kv - length + (min(r0 + m, rows) - 1) // G
                        shim.tiles_of(lo, hi, sink, window, cut, 1 << 24, out)
                        assert out[0] <= keys
                    shim.share(m, log_m, row_lo, row_hi, span, G, length, 0, cut, kv, 2, sink, window, out)
                    keys = out[1]
                    assert keys == (cut if out[0] else 0) if not window else keys <= cut
                    for pos in (64 * cut, 64 * cut + 1, 64 * cut + 63, 64 * cut + 500) if out[0] else ():      # rows behind the common part
                        shim.tiles_of(pos, pos + 70, sink, window, 0, cut, out)
                        assert out[0] <= keys


@pytest.mark.parametrize("name,least", [("paged_shared_merge_kernel", 4), ("paged_cut_kernel", 2), ("paged_append_q8", 4), ("paged_read_kernel", 2),
                                        ("paged_common_kernel", 1), ("paged_groups_kernel", 1)])
def test_no_kernel_uses_scratch(kernels, name, least):  # noqa: F811
    found = {n: k for n, k in kernels.items() if name in n}
    assert len(found) >= least
    for n, k in found.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n
