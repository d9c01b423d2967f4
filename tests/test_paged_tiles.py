"""CPU run of the index arithmetic by which the matrix kernels of the paged calls find their tiles and copy keys (csrc/pages.h, csrc/mask.h), over
wild tables and lengths: no copy leaves the pages, no table entry outside the row is looked at, every visible key is copied, every row is in one
tile."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

TILES = r"""
#include <climits>
#include <cstdio>
#include <initializer_list>
#include <random>
#include <vector>
#include "pages.h"
using namespace cf;

static int fail(const char *what, int a, int b, int c) { return std::printf("%s: %d %d %d\n", what, a, b, c), 1; }

struct Call {
    int columns, shift, n_pages, G;
    WindowMask mask;
    std::vector<int> cu, kv;
    std::vector<std::vector<int>> table;
};

// A copy of rows [0, least(size - 1, room)] of the group at `key`, and where a kernel says that they stand.
static int copy(const Call &c, const KeyPlaces &at, int entry, int key, int size, int room, std::vector<char> &copied)
{
    if (room < 0) return fail("room", key, size, room);
    const int64_t row_bytes = 6, page_bytes = 1000000007;        // (nothing that the arithmetic could cancel)
    const int64_t where = at.offset(entry, key, page_bytes, (unsigned)row_bytes);
    for (int r = 0; r < size; ++r) {
        const int row = at_most(r, room);
        const int64_t bytes = where + row * row_bytes, page = bytes / page_bytes, in_page = bytes % page_bytes / row_bytes;
        if (page != entry || page < 0 || page >= c.n_pages || in_page < 0 || in_page >= 1 << c.shift) return fail("outside the pages", key, r, entry);
        if (key + row < 0 || key + row > at.last) return fail("behind the last key", key, r, at.last);
        if (in_page != ((key + row) & ((1 << c.shift) - 1))) return fail("another row", key, r, (int)in_page);
        if (r <= room) copied[key + row] = 1;
    }
    return 0;
}

// All tiles of a call in tiles of BM rows; TILE: keys of a key tile; group: keys of a copy (a whole tile where it has its keys, else 16).
template <int BM, int TILE>
static int run(const Call &c, int group)
{
    const int n_seqs = (int)c.kv.size(), T = c.cu[n_seqs];
    const int64_t places = places_most(T, n_seqs, c.G, BM);
    std::vector<char> done((size_t)T * c.G, 0);
    for (int place = 0; place < places; ++place) {
        int seq = 0;
        for (int g = 0; g < n_seqs; ++g)
            if (first_place(c.cu[g], g, c.G, BM) <= place) seq = g;
        const NewRows rows(c.cu[seq], c.cu[seq + 1], c.kv[seq]);
        const TileSpan span(place, c.cu[seq], rows.lq, seq, c.G, BM);
        if (span.rows <= 0) continue;
        if (span.row0 < 0 || span.rows > BM) return fail("tile", place, span.row0, span.rows);
        auto position = [&](int x) { return at_least(-1, rows.first_position + (span.row0 + x) / c.G); };
        for (int x = 0; x < span.rows; ++x) {
            const int64_t at = (int64_t)(rows.q0 + (span.row0 + x) / c.G) * c.G + (span.row0 + x) % c.G;
            if (at < 0 || at >= (int64_t)T * c.G || done[at]++) return fail("row", place, x, (int)at);
            if (position(x) != rows.position((span.row0 + x) / c.G)) return fail("position", place, x, position(x));
        }
        const int lowest = position(0), highest = position(span.rows - 1), keys = keys_within(highest, c.columns, c.shift);
        const KeyTiles<TILE, WindowMask> tiles(c.mask, lowest, keys);
        const KeyPlaces at{c.shift, c.n_pages, keys - 1};
        std::vector<char> copied((size_t)at_least(0, keys), 0);
        for (int t = 0; t < tiles.n; ++t) {
            const int start = tiles.start(t);
            if (start < 0 || start >= keys) return fail("tile of keys", t, start, keys);
            for (int key = start; key < start + TILE; key += group) {
                const int column = at.column(key), entry = c.table[seq].at(column);
                if (at.none(entry, key)) continue;
                if (int rc = copy(c, at, entry, key, group, at.room(key), copied)) return rc;
            }
        }
        for (int x = 0; x < span.rows; ++x) {
            const int p = position(x);
            for (int j = 0; j <= p && j < keys; ++j) {
                const int entry = c.table[seq].at(j >> c.shift);
                const bool seen = ((int64_t)j > (int64_t)p - c.mask.window || j < c.mask.sinks) && entry >= 0 && entry < c.n_pages;
                if (seen && !copied[j]) return fail("missing key", place, x, j);
                if (copied[j] && !(entry >= 0 && entry < c.n_pages)) return fail("hidden page", place, x, j);
            }
        }
    }
    for (char d : done)
        if (d != 1) return fail("rows without a tile", d, 0, 0);
    return 0;
}

int main()
{
    std::mt19937 rng(7);
    auto pick = [&](std::initializer_list<int> a) { return a.begin()[rng() % a.size()]; };
    for (int n = 0; n < 3000; ++n) {
        Call c;
        c.shift = pick({4, 4, 5, 6, 7}), c.columns = pick({1, 2, 3, 7}), c.n_pages = pick({1, 5, 1000}), c.G = pick({1, 2, 3, 7, 16, 40});
        const int capacity = c.columns << c.shift, window = pick({0, 0, 1, 5, 16, 33, 64, 100, 500, INT_MAX}), sinks = pick({0, 1, 16, 17, 70, INT_MAX});
        c.mask = window == 0 ? WindowMask{INT_MAX, 0} : WindowMask{window, at_most(sinks, capacity)};
        c.cu = {0};
        for (int g = pick({1, 1, 2, 5}); g > 0; --g) {
            c.cu.push_back(c.cu.back() + pick({0, 0, 1, 1, 2, 9, 40}));
            c.kv.push_back(pick({INT_MIN, -1, 0, 1, 15, 16, 17, 33, 64, 100, capacity - 1, capacity, capacity + 1, capacity + 90, INT_MAX - 70, INT_MAX}));
            c.table.emplace_back();
            for (int x = 0; x < c.columns; ++x)
                c.table.back().push_back(pick({0, 0, (int)(rng() % c.n_pages), (int)(rng() % c.n_pages), c.n_pages - 1, c.n_pages, -1, INT_MIN, INT_MAX}));
        }
        if (c.cu.back() == 0) c.cu.back() = 1;
        // bf16: tiles of many rows and of few, key tiles of 64 in groups of 16 or, in pages that hold them, of 32 and whole; fp32: blocks of 16
        if (run<128, 64>(c, 16) || run<32, 64>(c, 16) || run<16, 16>(c, 16)) return 1;
        if (c.shift >= 6 && (run<128, 64>(c, 64) || run<32, 64>(c, 32))) return 1;
    }
    return 0;
}
"""


def test_no_copy_of_the_matrix_kernels_leaves_the_pages(tmp_path):
    src = tmp_path / "tiles.cpp"
    src.write_text(TILES)
    exe = str(tmp_path / "tiles")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined,address", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2503_02356_amd", "csrc"), str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr[-2000:]
