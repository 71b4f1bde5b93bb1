"""CPU tests of the paged cache's host side: the index arithmetic that the kernels run (csrc/paged_index.h) against brute force, page ids that no cache
has among it, and the library's refusals, which come before anything is launched."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import paper_2507_11978_amd as nt
from paper_2507_11978_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "paged_index.h"
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
using namespace nt;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main()
{
    std::mt19937_64 r(7);
    auto in = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(r() % (uint64_t)(hi - lo + 1)); };
    // division by every small divisor and by drawn ones, at multiples and beside them
    for (int i = 0; i < 4000; ++i) {
        const uint32_t d = i < 2000 ? i + 1 : (uint32_t)in(1, 1 << 24);
        const Divider v = divider_of(d);
        for (int j = 0; j < 200; ++j) {
            const uint32_t q = (uint32_t)in(0, 0x7fffffff / d), n[3] = {q * d, q ? q * d - 1 : 0, (uint32_t)in(0, 0x7fffffff)};
            for (uint32_t x : n) CHECK(divide(x, v) == x / d);
        }
        CHECK(divide(0x7fffffff, v) == 0x7fffffffu / d);
    }
    // table entries: only pages that exist come through, and nothing past the row's end is read
    for (int i = 0; i < 2000; ++i) {
        const int width = (int)in(0, 9), pages = (int)in(0, 5);
        std::vector<int32_t> row(width);
        const int32_t odd[] = {-1, INT32_MIN, INT32_MAX, pages, pages + 1, -2};
        for (int32_t &e : row) e = in(0, 2) ? (int32_t)in(0, 5) : odd[in(0, 5)];
        for (uint32_t k : {0u, 1u, 5u, (uint32_t)width, 0x7fffffffu, 0xffffffffu}) {
            const int32_t got = page_at(row.data(), k, width, pages);
            const bool has = k < (uint32_t)width && row[k] >= 0 && row[k] < pages;
            CHECK(got == (has ? row[k] : -1));
        }
    }
    // sequences: rows stay inside the queries whatever the arrays hold
    for (int i = 0; i < 20000; ++i) {
        const int32_t T = (int32_t)in(0, 50), s[2] = {(int32_t)in(-60, 60), (int32_t)in(-60, 60)}, n[1] = {(int32_t)in(-3, 60)};
        const Sequence q = sequence_at(s, n, 0, T);
        CHECK(q.first >= 0 && q.count >= 0 && q.first + q.count <= T && q.length >= 0);
        if (0 <= s[0] && s[0] <= s[1] && s[1] <= T) CHECK(q.first == s[0] && q.count == s[1] - s[0]);
    }
    // the keys of a tile and its shares: what some token sees, each key in one share, shares beginning at multiples of the block
    for (int i = 0; i < 20000; ++i) {
        const int32_t count = (int32_t)in(1, 40), length = (int32_t)in(0, 200), causal = (int32_t)in(0, 1), window = in(0, 1) ? (int32_t)in(1, 90) : 0;
        const Sequence q{0, count, length};
        const int32_t i0 = (int32_t)in(0, count - 1), i1 = (int32_t)in(i0, count - 1), block = in(0, 1) ? 32 : 64, splits = (int32_t)in(1, 5), share = block * (int32_t)in(1, 3);
        std::vector<int> seen(201, 0), taken(201, 0);
        for (int t = i0; t <= i1; ++t) {
            const int64_t pos = (int64_t)length - count + t;
            const KeyRange k = keys_seen(q, t, causal, window);
            for (int64_t j = 0; j < length; ++j) {
                const bool sees = (!causal || j <= pos) && (!window || j > pos - window);
                CHECK(sees == (j >= k.lo && j < k.hi));
                seen[j] |= sees;
            }
        }
        for (int s = 0; s < splits; ++s) {
            const KeyRange k = key_range(q, i0, i1, causal, window, s, splits, share, block);
            CHECK(0 <= k.lo && k.lo <= k.hi && k.hi <= length);
            if (s > 0 && k.lo < k.hi) CHECK(k.lo % block == 0);
            for (int j = k.lo; j < k.hi; ++j) ++taken[j];
        }
        for (int j = 0; j <= length; ++j) CHECK(taken[j] <= 1 && (!seen[j] || taken[j] == 1));
    }
    // tile numbers: each sequence has room for its rows, and all of them fit the grid
    for (int i = 0; i < 5000; ++i) {
        const int B = (int)in(1, 9), group = (int)in(1, 20), rows = 128;
        std::vector<int32_t> starts(B + 1, 0);
        for (int b = 0; b < B; ++b) starts[b + 1] = starts[b] + (int32_t)(in(0, 2) ? in(0, 60) : 0);
        const int32_t T = starts[B];
        for (int b = 0; b < B; ++b) {
            const int32_t need = ((starts[b + 1] - starts[b]) * group + rows - 1) / rows, at = first_tile(starts.data(), b, T, group, rows);
            const int64_t next = b + 1 < B ? first_tile(starts.data(), b + 1, T, group, rows) : (int64_t)T * group / rows + B;
            CHECK(at + need <= next);
        }
    }
    puts("good");
}
"""


def test_index_arithmetic(tmp_path):
    (tmp_path / "t.cpp").write_text(PROGRAM)
    csrc = os.path.join(ROOT, "paper_2507_11978_amd", "csrc")
    subprocess.run(["g++", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-std=c++17", "-I", csrc, str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")], check=True)
    out = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "good", out.stdout + out.stderr


# ---- refusals, on made-up addresses: nothing is launched
F16, BF16, F32, E4M3, I8 = range(5)
ADDRESS = 1 << 40


def cache(pages=4, page=16, heads=2, size=64, dtype=F16, scales=False, **over):
    shape = (pages, page, heads, size)
    a = dict(k=ADDRESS, v=ADDRESS, dk=binding.make_desc(shape), dv=binding.make_desc(shape), dtype=dtype)
    if scales:
        a.update(k_scale=ADDRESS, v_scale=ADDRESS, dks=binding.make_desc(shape[:3]), dvs=binding.make_desc(shape[:3]))
    a.update(over)
    c = binding.PagedCache(dtype=a["dtype"], k=a["k"], v=a["v"], k_scale=a.get("k_scale"), v_scale=a.get("v_scale"))
    for name in ("dk", "dv", "dks", "dvs"):
        if a.get(name) is not None:
            setattr(c, name, C.pointer(a[name]))
    return c


def moved(write, c, tokens=(3, 2, 64), tokens_v=None, dtype=F16, k=ADDRESS, slots=ADDRESS):
    dk, dv = (d if isinstance(d, binding.TensorDesc) else binding.make_desc(d) for d in (tokens, tokens_v or tokens))
    fn = binding.load().nt_cache_write if write else binding.load().nt_cache_read
    st = fn(C.byref(c) if c is not None else None, k, C.byref(dk), ADDRESS, C.byref(dv), slots, dtype, None)
    return binding._STATUS.get(st, st), binding.load().nt_last_error().decode()


strided = binding.make_desc((4, 16, 2, 64), (2 * 16 * 2 * 64, 2 * 2 * 64, 2 * 64, 2))
BAD_CACHES = [
    (dict(k=None), "NT_ERR_INVALID_ARG", "null device pointer"),
    (dict(dk=None), "NT_ERR_INVALID_ARG", "null cache or descriptor"),
    (dict(dk=binding.make_desc((4, 16, 2))), "NT_ERR_SHAPE_MISMATCH", "4-D"),
    (dict(dv=binding.make_desc((4, 16, 2, 72))), "NT_ERR_SHAPE_MISMATCH", "differ in size"),
    (dict(dk=strided, dv=strided), "NT_ERR_UNSUPPORTED", "unit stride"),
    (dict(size=60), "NT_ERR_UNSUPPORTED", "multiple of 8"),
    (dict(size=264), "NT_ERR_UNSUPPORTED", "multiple of 8"),
    (dict(page=0), "NT_ERR_UNSUPPORTED", "page_size"),
    (dict(heads=0), "NT_ERR_UNSUPPORTED", "heads"),
    (dict(dtype=BF16), "NT_ERR_UNSUPPORTED", "the tokens' type"),
    (dict(dtype=F32), "NT_ERR_UNSUPPORTED", "the tokens' type"),
    (dict(dtype=E4M3), "NT_ERR_INVALID_ARG", "needs scales"),
    (dict(scales=True), "NT_ERR_INVALID_ARG", "8-bit caches only"),
    (dict(dtype=I8, scales=True, dks=binding.make_desc((4, 16, 2, 1))), "NT_ERR_SHAPE_MISMATCH", "3-D"),
    (dict(dtype=I8, scales=True, dvs=binding.make_desc((4, 16, 3))), "NT_ERR_SHAPE_MISMATCH", "differ in size"),
    (dict(dtype=I8, scales=True, k_scale=None), "NT_ERR_INVALID_ARG", "null device pointer"),
]


@pytest.mark.parametrize("write", [True, False])
def test_cache_refusals(write):
    for over, name, text in BAD_CACHES:
        got = moved(write, cache(**over))
        assert got[0] == name and text in got[1], (over, got)
    for args, name, text in [
            (dict(tokens=(3, 2, 64), tokens_v=(4, 2, 64)), "NT_ERR_SHAPE_MISMATCH", "K and V differ"),
            (dict(tokens=(3, 3, 64)), "NT_ERR_SHAPE_MISMATCH", "heads or head_size"),
            (dict(tokens=(3, 2, 56)), "NT_ERR_SHAPE_MISMATCH", "heads or head_size"),
            (dict(tokens=(3, 2)), "NT_ERR_SHAPE_MISMATCH", "3-D"),
            (dict(tokens=binding.make_desc((3, 2, 64), (256, 128, 2))), "NT_ERR_UNSUPPORTED", "unit stride"),
            (dict(tokens=(1 << 30, 2, 64)), "NT_ERR_UNSUPPORTED", "2^31"),
            (dict(dtype=F32), "NT_ERR_UNSUPPORTED", "dtype"),
            (dict(k=None), "NT_ERR_INVALID_ARG", "null device pointer"),
            (dict(slots=None), "NT_ERR_INVALID_ARG", "null device pointer")]:
        got = moved(write, cache(), **args)
        assert got[0] == name and text in got[1], (args, got)
    assert moved(write, None)[0] == "NT_ERR_INVALID_ARG"
    assert moved(write, cache(), tokens=(0, 2, 64), k=None, slots=None)[0] == 0          # no tokens: nothing to do


def attended(c, q=(5, 4, 64), out=None, table=(2, 3), dtype=F16, scale=0.0, window=0, max_queries=0, max_length=0, pq=ADDRESS, starts=ADDRESS, pt=ADDRESS):
    dq, do, dt = (d if isinstance(d, binding.TensorDesc) else binding.make_desc(d) for d in (q, out or q, table))
    st = binding.load().nt_sdpa_paged(pq, C.byref(dq), C.byref(c), pt, C.byref(dt), starts, ADDRESS, ADDRESS, C.byref(do), scale, 1, window, max_queries,
                                      max_length, dtype, None)
    return binding._STATUS.get(st, st), binding.load().nt_last_error().decode()


def test_attention_refusals():
    for over, name, text in BAD_CACHES:
        got = attended(cache(**over))
        assert got[0] == name and text in got[1], (over, got)
    for args, name, text in [
            (dict(q=(5, 4)), "NT_ERR_SHAPE_MISMATCH", "3-D"),
            (dict(q=(5, 4, 64), out=(5, 4, 72)), "NT_ERR_SHAPE_MISMATCH", "queries and output"),
            (dict(q=(5, 4, 72)), "NT_ERR_SHAPE_MISMATCH", "head_size"),
            (dict(q=(5, 3, 64)), "NT_ERR_SHAPE_MISMATCH", "multiple of the cache's heads"),
            (dict(q=(5, 0, 64)), "NT_ERR_SHAPE_MISMATCH", "multiple of the cache's heads"),
            (dict(q=binding.make_desc((5, 4, 64), (512, 128, 2))), "NT_ERR_UNSUPPORTED", "unit stride"),
            (dict(table=(2, 3, 1)), "NT_ERR_SHAPE_MISMATCH", "2-D"),
            (dict(table=binding.make_desc((2, 3), (6, 2))), "NT_ERR_UNSUPPORTED", "unit stride"),
            (dict(scale=float("nan")), "NT_ERR_INVALID_ARG", "NaN"),
            (dict(window=-1), "NT_ERR_INVALID_ARG", "negative"),
            (dict(max_queries=-1), "NT_ERR_INVALID_ARG", "negative"),
            (dict(max_length=-5), "NT_ERR_INVALID_ARG", "negative"),
            (dict(q=(1 << 29, 4, 64)), "NT_ERR_UNSUPPORTED", "2^30"),
            (dict(dtype=F32), "NT_ERR_UNSUPPORTED", "dtype"),
            (dict(pq=None), "NT_ERR_INVALID_ARG", "null device pointer"),
            (dict(starts=None), "NT_ERR_INVALID_ARG", "null device pointer"),
            (dict(pt=None), "NT_ERR_INVALID_ARG", "null device pointer")]:
        got = attended(cache(), **args)
        assert got[0] == name and text in got[1], (args, got)
    assert attended(cache(pages=0, k=None, v=None))[0] == "NT_ERR_INVALID_ARG"           # tokens, but no pages
    assert attended(cache(), q=(0, 4, 64), pq=None)[0] == 0
    assert attended(cache(), table=(0, 3))[0] == 0
    assert nt.last_paged_plan().rows == 0


def test_tensors_off_the_gpu_and_of_other_types_are_refused():
    k = torch.zeros(3, 2, 64, dtype=torch.float16)
    c = torch.zeros(4, 16, 2, 64, dtype=torch.float16)
    slots = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        nt.cache_write(k, k, slots, c, c)
    with pytest.raises(ValueError):
        nt.cache_read(c, c, slots, k, k)
    with pytest.raises(ValueError):
        nt.sdpa_paged(k, c, c, torch.zeros(1, 1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.empty_like(k))
