"""CPU tests of lengths that no cache has (csrc/paged_index.h): what the paged attention kernels walk and look up stays within the table's reach and 32 bits,
and every token that sees a position without a table entry still meets one."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "paged_index.h"
#include <algorithm>
#include <cstdio>
#include <random>
using namespace nt;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main()
{
    std::mt19937_64 r(11);
    auto in = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(r() % (uint64_t)(hi - lo + 1)); };
    // small ones, against brute force: tokens i0 .. i1 of a sequence, a table with room for `capacity` positions
    for (int i = 0; i < 40000; ++i) {
        const int32_t count = (int32_t)in(1, 30), length = (int32_t)in(0, 150), causal = (int32_t)in(0, 1), window = in(0, 1) ? (int32_t)in(1, 70) : 0;
        const int32_t capacity = (int32_t)in(0, 160), i0 = (int32_t)in(0, count - 1), i1 = (int32_t)in(i0, count - 1), block = in(0, 1) ? 32 : 64;
        const int32_t splits = (int32_t)in(1, 4), share = block * (int32_t)in(1, 3);
        const Sequence q{0, count, length};
        bool walked[152] = {};
        int64_t keys = 0;
        for (int s = 0; s < splits; ++s) {
            const KeyRange k = key_range(q, i0, i1, causal, window, s, splits, share, block, capacity);
            CHECK(0 <= k.lo && k.lo <= k.hi && k.hi <= length);
            for (int j = k.lo; j < k.hi; ++j) {
                CHECK(!walked[j]);
                walked[j] = true;
            }
            keys += k.hi - k.lo;
        }
        CHECK(keys <= capacity + (i1 - i0) + 1);
        for (int t = i0; t <= i1; ++t) {
            const KeyRange k = keys_seen(q, t, causal, window);
            bool beyond = false, met = false;
            for (int j = std::max(0, k.lo); j < k.hi; ++j) {
                beyond |= j >= capacity;
                met |= j >= capacity && walked[j];
                CHECK(j >= capacity || walked[j]);
            }
            CHECK(beyond == met);
        }
    }
    // the largest: whatever the arrays hold, the blocks of the range and the three thousand keys behind it have numbers below 2^31, places on their pages
    // and, where they have one, an entry of the table
    for (int i = 0; i < 200000; ++i) {
        const int32_t T = (int32_t)in(1, 1 << 20), starts[2] = {0, T}, lengths[1] = {(int32_t)(INT32_MAX - (in(0, 3) ? in(0, 9000) : in(0, INT32_MAX)))};
        const Sequence q = sequence_at(starts, lengths, 0, T);
        CHECK(q.length == std::min(lengths[0], kMostKeys + 1));
        const uint32_t page = (uint32_t)(in(0, 1) ? in(1, 1 << 24) : (1 << in(0, 24)) - (in(0, 1) ? 1 : 0));
        if (!page) continue;
        const int64_t W = in(0, 1) ? in(0, INT32_MAX) : in(0, 100);
        const int32_t width = entries_in_reach(W, page);
        CHECK(width <= W && (int64_t)width * page <= kMostKeys && (width == W || (int64_t)(width + 1) * page > kMostKeys));
        const int32_t capacity = (int32_t)(width * page), causal = (int32_t)in(0, 1), window = in(0, 2) ? (int32_t)in(1, 1 << in(1, 30)) : 0, t = (int32_t)in(0, T - 1);
        const KeyRange k = key_range(q, t, std::min(t + 127, T - 1), causal, window, 0, 1, 64, 64, capacity);
        CHECK(0 <= k.lo && k.lo <= k.hi && k.hi <= kMostKeys + 1);
        const Divider d = divider_of(page);
        for (int j = 0; j < 8; ++j) {
            const int64_t key = j < 4 ? k.hi - 1 + in(0, 3000) : in(k.lo, (int64_t)k.hi + 3000);
            CHECK(key <= INT32_MAX);
            const uint32_t index = divide((uint32_t)key, d);
            CHECK(index == key / page && (index < (uint32_t)width) == (key < capacity));
        }
    }
    // windows of any length
    for (int i = 0; i < 200000; ++i) {
        const int32_t count = (int32_t)in(1, 1 << 30), length = (int32_t)in(0, kMostKeys + 1), window = (int32_t)(INT32_MAX - (in(0, 1) ? in(0, 1 << 20) : in(0, INT32_MAX - 1)));
        const Sequence q{0, count, length};
        const int32_t t = (int32_t)in(0, count - 1);
        const KeyRange k = keys_seen(q, t, 1, window);
        const int64_t pos = (int64_t)length - count + t, lo = pos - window + 1;
        CHECK(k.hi == pos + 1 && (int64_t)(k.lo > 0 ? k.lo : 0) == (lo > 0 ? lo : 0));
    }
    puts("good");
}
"""


def test_lengths_beyond_any_cache(tmp_path):
    (tmp_path / "t.cpp").write_text(PROGRAM)
    csrc = os.path.join(ROOT, "paper_2507_11978_amd", "csrc")
    subprocess.run(["g++", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-std=c++17", "-I", csrc, str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")], check=True)
    out = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "good", out.stdout + out.stderr
