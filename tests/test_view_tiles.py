"""Which tiles the calls through sliding windows walk and request, checked with the kernels' own functions, compiled for the
host (no GPU is touched): every tile is one of the sequence's, each that holds a token which is seen comes once, and what is
requested for a walk without tiles (a split that lies behind a shorter view, a block behind the last row) is one of them too."""
import ctypes
import itertools
import os
import subprocess

import pytest

from paper_2405_03917_amd import build as cq_build

PROBE = r"""
#include <vector>

#include "cq_decode_split.hpp"
#include "cq_lds_gather.hpp"
namespace cq {
// 0, or the number of the first rule that does not hold
template <class View, class Sees>
int walk(const View& view, int most, int last, Sees&& sees)
{
    if (view.n_tiles < 1 || view.n_tiles > most) return 1;
    std::vector<char> walked(last / kTileTokens + 1, 0);
    for (int i = 0; i < view.n_tiles; ++i) {
        const int tile = view.tile(i);
        if (tile < 0 || tile > last / kTileTokens) return 2;
        if (walked[tile]++) return 3;
    }
    for (int tok = 0; tok <= last; ++tok)
        if (sees(tok) && !walked[tok / kTileTokens]) return 4;
    return 0;
}

// Decode: a sequence of t_n of up to t tokens.
extern "C" __attribute__((visibility("default"))) int decode_view(int t, int t_n, int window, int n_sink)
{
    DecodeViewArgs a;
    a.t = t;
    a.window = window;
    a.n_sink = n_sink;
    const Seen<kWindow> seen(a, t_n);
    if (const int bad = walk(seen, view_tiles(t, 1, window, n_sink), t_n - 1, [&](int tok) { return seen.token(tok, t_n); })) return bad;
    for (int i = 0; i < seen.n_tiles; ++i) {
        int n = 0;
        for (int u = 0; u < kTileTokens; ++u) n += seen.token(seen.tile(i) * kTileTokens + u, t_n);
        if (n == 0) return 5;                               // (a chunk's maximum is a score)
        if (n < kTileTokens && !seen.edge(i)) return 6;
    }
    return 0;
}

// Chunks: the rows of `block` rows each (those of a workgroup or of a wavefront), `blocks` of them, and splits of `tiles` tiles.
extern "C" __attribute__((visibility("default"))) int chunk_view(int t, int t_n, int m, int qper, int block, int blocks, int window, int n_sink, int tiles)
{
    ChunkViewArgs a;
    a.t = t;
    a.m = m;
    a.window = window;
    a.n_sink = n_sink;
    const int rows = m * qper, pos0 = t_n - m, most = view_tiles(t, m, window, n_sink), n_split = (most + tiles - 1) / tiles;
    for (int b = 0; b < blocks; ++b) {
        const int first = pos0 + (b * block < rows ? b * block : rows - 1) / qper;
        const int last = pos0 + ((b + 1) * block < rows ? (b + 1) * block - 1 : rows - 1) / qper;
        const ChunkSeen seen(a, first, last);
        if (const int bad = walk(seen, most, last, [&](int tok) {
                for (int p = first; p <= last; ++p)
                    if (in_window(a, tok, p)) return true;
                return false;
            }))
            return bad;
        for (int split = 0; split < n_split; ++split) {
            const int tile0 = split * tiles, end = tile0 + tiles < seen.n_tiles ? tile0 + tiles : seen.n_tiles;
            const int tile1 = b * block < rows ? end : tile0;
            for (int i = tile0; i < tile0 + tiles + 24; ++i) {      // (up to three rounds of eight wavefronts ahead)
                const int at = seen.requested(i, tile0, tile1);
                bool mine = false;
                for (int j = 0; j < seen.n_tiles; ++j) mine = mine || seen.tile(j) == at;
                if (at > (t_n - 1) / kTileTokens) return 7;
                if (!mine) return 8;
                if (i < tile1 && at != seen.tile(i)) return 9;
            }
        }
    }
    return 0;
}
}
"""


@pytest.fixture(scope="module")
def views(tmp_path_factory):
    if not os.path.exists(cq_build.HIPCC):
        pytest.skip("no hipcc")
    at = tmp_path_factory.mktemp("views")
    (at / "views.hip").write_text(PROBE)
    cmd = [cq_build.HIPCC, *cq_build.FLAGS, "--offload-host-only", "-shared", str(at / "views.hip"), "-o", str(at / "views.so")]
    done = subprocess.run(cmd, capture_output=True, text=True)
    assert done.returncode == 0, done.stderr[-3000:]
    return ctypes.CDLL(str(at / "views.so"))


LENGTHS = [1, 2, 63, 64, 65, 127, 128, 129, 448, 500, 1023, 1024]
WINDOWS = [1, 2, 63, 64, 65, 66, 100, 128, 192, 500, 1024]
SINKS = [0, 1, 4, 63, 64, 65, 200, 1024]


def test_decode_views(views):
    for t, t_n, window, sink in itertools.product([64, 500, 1024], LENGTHS, WINDOWS, SINKS):
        if t_n <= t and window <= t and sink <= t:
            assert views.decode_view(t, t_n, window, sink) == 0, (t, t_n, window, sink)


# rows of a wavefront of the kernel for few rows (one, two or four blocks of 16), of a workgroup of the one for many (128, 256)
@pytest.mark.parametrize("m,qper,block,blocks", [(1, 1, 16, 1), (3, 1, 16, 1), (5, 1, 16, 1), (10, 4, 16, 4), (11, 4, 16, 4), (16, 1, 16, 1), (17, 1, 16, 2),
                                                 (33, 1, 16, 4), (64, 1, 16, 4), (9, 7, 16, 4), (3, 1, 128, 1), (129, 1, 128, 2), (300, 2, 256, 3)])
def test_chunk_views_and_requests(views, m, qper, block, blocks):
    for t, t_n, window, sink, tiles in itertools.product([448, 1024], LENGTHS, WINDOWS, SINKS[:6], [1, 2, 9]):
        if m <= t_n <= t and window <= t:
            assert views.chunk_view(t, t_n, m, qper, block, blocks, window, sink, tiles) == 0, (t, t_n, window, sink, tiles)


@pytest.mark.parametrize("t,m,qper,blocks,window,sink", [(4096, 5, 1, 1, 1024, 4), (23872, 10, 4, 4, 5076, 4), (52608, 11, 4, 4, 7359, 64)])
def test_requests_of_full_caches(views, t, m, qper, blocks, window, sink):
    for tiles in range(1, 24):
        assert views.chunk_view(t, t, m, qper, 16, blocks, window, sink, tiles) == 0, tiles
