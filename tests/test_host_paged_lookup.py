"""CPU test of the paged attention kernels' page lookup (csrc/paged_index.h: entry_read, names_page), under the address sanitizer: no entry outside the table row is
read, and no page outside the cache is taken, whatever the position and whatever the table holds."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_11978_amd", "csrc")

PROGRAM = r"""
#include "paged_index.h"
#include <cstdio>
#include <memory>
#include <random>
using namespace nt;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main()
{
    std::mt19937_64 r(5);
    auto in = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(r() % (uint64_t)(hi - lo + 1)); };
    for (int i = 0; i < 20000; ++i) {
        const int32_t width = (int32_t)(i < 600 ? i % 3 : in(0, 40)), pages = (int32_t)in(1, 6);
        const uint32_t page_size = (uint32_t)(in(0, 3) ? in(1, 70) : in(1, 1 << 24));
        const int64_t held = width > 0 ? width : 1;                        // (a row without entries: the launcher has one number in its place)
        std::unique_ptr<int32_t[]> row(new int32_t[held]);
        const int32_t odd[] = {-1, INT32_MIN, INT32_MAX, pages, pages + 1, -2};
        for (int64_t e = 0; e < held; ++e) row[e] = in(0, 2) ? (int32_t)in(0, pages - 1) : odd[in(0, 5)];
        const Divider d = divider_of(page_size);
        const int64_t reach = (int64_t)width * page_size;
        for (int j = 0; j < 40; ++j) {
            int64_t key = j < 4 ? j : j < 20 ? reach + in(-3, 600) : j < 30 ? (int64_t)INT32_MAX - in(0, 4000) : in(0, reach);
            if (key < 0 || key > INT32_MAX) continue;
            const uint32_t index = divide((uint32_t)key, d), at = (uint32_t)key - index * page_size, entry = entry_read(index, width);
            CHECK(entry < (uint32_t)held);
            const int32_t id = row[entry];
            const bool named = names_page(index, id, width, pages);
            const bool want = key < reach && row[key / page_size] >= 0 && row[key / page_size] < pages;
            CHECK(named == want);
            const uint32_t page = named ? (uint32_t)id : 0;
            CHECK(page < (uint32_t)pages && at < page_size && (!named || (int64_t)page == row[key / page_size]));
        }
        for (uint32_t index : {0x80000000u, 0xffffffffu, (uint32_t)width}) CHECK(entry_read(index, width) < (uint32_t)held && !names_page(index, 0, width, pages));
    }
    puts("good");
}
"""


def test_page_lookup(tmp_path):
    (tmp_path / "t.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-std=c++17", "-I", CSRC, str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")], check=True)
    out = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "good", out.stdout + out.stderr


def test_the_kernels_have_no_other_lookup():
    """Every reading of a table row goes through entry_read, every use of what was read through names_page."""
    for name in ("paged_few.h", "paged_many.h"):
        with open(os.path.join(CSRC, name)) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        assert text.count("entry_read(") == (1 if name == "paged_few.h" else 2) and text.count("names_page(") == text.count("entry_read(")
        assert not re.search(r"<[^;]*\bg\.(width|pages)\b", text)
