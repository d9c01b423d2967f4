"""CPU run of the arithmetic of a cache of 8 bits (csrc/pages8.h): powers of two of the blocks, that every block which a call adds to has one place in
the launch, and only one, and every head of a pair one workgroup."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = r"""
#include <climits>
#include <cmath>
#include <cstdio>
#include <initializer_list>
#include <random>
#include <vector>
#include "pages8.h"
using namespace cf;

static int powers()
{
    std::mt19937 rng(3);
    auto one = [](float most) {
        const int e = exponent_for(most);
        if (e < kLeast8 || e > kMost8 || (double)most > std::ldexp(448.0, e)) return std::printf("%a: 2^%d is too small\n", most, e), 1;
        if (e > kLeast8 && (double)most <= std::ldexp(448.0, e - 1)) return std::printf("%a: 2^%d is not the least\n", most, e), 1;
        return 0;
    };
    for (int e = -149; e <= 127; ++e)
        for (double f : {1.0, 1.75, 1.9999, 1.5}) {
            const float x = (float)std::ldexp(f, e);
            if (std::isinf(x)) continue;
            if (one(x) || one(std::nextafterf(x, 0.f))) return 1;
            if (std::isfinite(std::nextafterf(x, INFINITY)) && one(std::nextafterf(x, INFINITY))) return 1;
        }
    if (one(0.f) || exponent_for(0.f) != kLeast8 || one(3.402823466e38f)) return 1;
    for (int i = 0; i < 100000; ++i) {
        const float x = float_of(rng() & 0x7fffffff);
        if (std::isfinite(x) && one(x)) return 1;
    }
    for (int e = kLeast8; e <= kMost8; ++e)
        if (power8(e) != std::ldexp(1.f, e) || exponent_of(power8(e)) != e || factor8(power8(e)) != power8(e) || power8(-e) * power8(e) != 1.f) return std::printf("2^%d\n", e), 1;
    // whatever stands in the pages
    for (float x : {0.f, -1.5f, 3.f, INFINITY, -INFINITY, NAN, 1e-45f, 3e38f})
        if (exponent_of(x) < -127 || exponent_of(x) > 128 || (exponent_of(x) < 128 && factor8(x) != std::ldexp(1.f, exponent_of(x)))) return 1;
    for (int e = kLeast8; e <= 127; ++e)
        if (inverse8(e) != std::ldexp(1.f, -e)) return std::printf("2^-%d\n", e), 1;
    if (inverse8(128) != std::ldexp(1.f, -127)) return 1;
    return factor8(3.f) == 2.f && factor8(-1.5f) == 1.f && factor8(0.f) == std::ldexp(1.f, -127) && std::isnan(factor8(INFINITY)) && std::isnan(factor8(NAN)) ? 0 : 1;
}

static int places()
{
    std::mt19937 rng(5);
    auto pick = [&](std::initializer_list<int> a) { return a.begin()[rng() % a.size()]; };
    for (int n = 0; n < 20000; ++n) {
        std::vector<int> cu{0}, kv;
        for (int g = pick({1, 1, 2, 5, 30}); g > 0; --g) {
            cu.push_back(cu.back() + pick({0, 0, 1, 1, 2, 15, 16, 17, 31, 33, 100}));
            kv.push_back(pick({INT_MIN, -1, 0, 1, 2, 15, 16, 17, 18, 31, 32, 33, 100, 1000, INT_MAX - 20, INT_MAX}));
        }
        const int n_seqs = (int)kv.size(), T = cu.back();
        std::vector<char> done(T, 0);
        BlockPlaces places(T, n_seqs);
        if (places.all(T, n_seqs) != (T < T / 16 + 2 * n_seqs ? T : T / 16 + 2 * n_seqs)) return std::printf("places %d %d\n", T, n_seqs), 1;
        if (n % 2) places.of_rows = rng() % 2;       // (either way is right for any call)
        for (int place = 0; place < places.all(T, n_seqs); ++place) {
            int seq = 0;
            for (int g = 0; g < n_seqs; ++g)
                if (places.first(cu[g], g) <= place) seq = g;
            const NewRows rows(cu[seq], cu[seq + 1], kv[seq]);
            const NewBlocks blocks(rows);
            const int x = place - places.first(cu[seq], seq);
            if (x < 0) return std::printf("place %d\n", place), 1;
            if (x >= blocks.n) continue;
            const int key0 = (blocks.first + x) * kBlock8;
            int some = 0;
            for (int64_t key = key0; key < (int64_t)key0 + kBlock8; ++key) {
                if (key < blocks.begin || key >= blocks.end) continue;
                const int64_t row = (int64_t)rows.q0 + key - rows.first_position;
                if (row < cu[seq] || row >= cu[seq + 1] || done[row]++) return std::printf("row %d\n", (int)row), 1;
                if (rows.position((int)row - rows.q0) != key) return std::printf("position of row %d\n", (int)row), 1;
                ++some;
            }
            if (!some) return std::printf("a block of no rows\n"), 1;
        }
        for (int g = 0; g < n_seqs; ++g)
            for (int r = cu[g]; r < cu[g + 1]; ++r)
                if (done[r] != (NewRows(cu[g], cu[g + 1], kv[g]).position(r - cu[g]) >= 0)) return std::printf("row %d of %d: %d\n", r, g, done[r]), 1;
    }
    return 0;
}

static int pairs()
{
    for (int all = 2; all < 200; all += 2) {
        std::vector<int> done(all, 0);
        for (int id = 0; id < all; ++id) {
            const HeadPair p(id, all);
            if (p.pair < 0 || p.pair >= all / 2 || p.second < 0 || p.second > 1 || done[2 * p.pair + p.second]++) return std::printf("%d of %d: pair %d, %d\n", id, all, p.pair, p.second), 1;
            if (id < (all & ~15) && p.second) {
                const HeadPair q(id - 8, all);
                if (q.pair != p.pair || q.second) return std::printf("%d of %d: not beside %d\n", id, all, id - 8), 1;
            }
        }
    }
    return 0;
}

int main() { return powers() || places() || pairs(); }
"""


def test_powers_and_places(tmp_path):
    src = tmp_path / "pages8.cpp"
    src.write_text(CODE)
    exe = str(tmp_path / "pages8")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined,address", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2503_02356_amd", "csrc"), str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr[-2000:]
