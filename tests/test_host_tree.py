"""CPU tests of the host side of drafted tokens over a paged cache: which keys a tree's rows see and a program walks (csrc/paged_index.h) against brute force, and the
library's refusals, which come before anything is launched."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import paper_2507_11978_amd as nt
from paper_2507_11978_amd import binding
from test_host_paged import ADDRESS, BAD_CACHES, BF16, E4M3, F16, F32, I8, ROOT, cache

PROGRAM = r"""
#include "paged_index.h"
#include <cstdio>
#include <random>
#include <vector>
using namespace nt;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main()
{
    std::mt19937_64 r(5);
    auto in = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(r() % (uint64_t)(hi - lo + 1)); };
    for (int i = 0; i < 4000; ++i) {
        const int32_t a = (int32_t)in(-70, 70), b = (int32_t)in(-70, 70);
        const uint64_t m = bits_between(a, b);
        for (int j = 0; j < 64; ++j) CHECK(((m >> j) & 1) == (j >= a && j < b));
        std::vector<uint64_t> words(in(1, 4));                              // (their end is guarded)
        for (uint64_t &w : words) w = r();
        const int32_t at = in(0, 3) ? (int32_t)in(-130, 330) : (int32_t)(in(0, 1) ? in(INT32_MIN, -1000) : in(1000, INT32_MAX));
        const uint64_t got = bits_from(words.data(), (int32_t)words.size(), at);
        for (int j = 0; j < 64; ++j) {
            const int64_t k = (int64_t)at + j;
            const bool bit = k >= 0 && k < 64 * (int64_t)words.size() && ((words[k / 64] >> (k % 64)) & 1);
            CHECK(((got >> j) & 1) == bit);
        }
    }
    // rows: every key of every block
    for (int i = 0; i < 20000; ++i) {
        const int32_t count = (int32_t)in(1, 150), length = (int32_t)in(0, 300), window = in(0, 1) ? (int32_t)in(1, 200) : 0, depth = (int32_t)in(-2, 160);
        const int32_t words = (int32_t)in(1, 3), past = length - count, lo = tree_row_lo(past, count, depth, window);
        const int32_t d = depth < 0 ? 0 : depth > count - 1 ? count - 1 : depth;
        std::vector<uint64_t> mask(words);
        for (uint64_t &w : mask) w = r();
        for (int32_t base = 0; base < length; base += 32) {
            const uint64_t got = tree_keys(mask.data(), words, base, lo, past, length);
            for (int j = 0; j < 64; ++j) {
                const int32_t key = base + j, k = key - past;
                bool sees = false;
                if (key < past) sees = !window || key > past + d - window;
                else if (key < length && k >= 0 && k < 64 * words) sees = (mask[k / 64] >> (k % 64)) & 1;
                CHECK(((got >> j) & 1) == sees);
            }
        }
    }
    // ... near the largest positions, where sums must not wrap
    for (int i = 0; i < 2000; ++i) {
        const int32_t count = (int32_t)in(1, 130), length = kMostKeys + 1 - (int32_t)in(0, 70), past = length - count, base = (int32_t)in(past - 140, length - 1);
        std::vector<uint64_t> mask(3);
        for (uint64_t &w : mask) w = r();
        const uint64_t got = tree_keys(mask.data(), 3, base, 0, past, length);
        for (int64_t j = 0; j < 64; ++j) {
            const int64_t key = base + j, k = key - past;
            CHECK(((got >> j) & 1) == (key < past || (key < length && ((mask[k / 64] >> (k % 64)) & 1))));
        }
        CHECK(tree_row_lo(past, count, count - 1, 1) == past && tree_row_lo(past, count, 0, INT32_MAX) == (past >= INT32_MAX ? 1 : 0));
    }
    // what the programs of a sequence walk: all that some token may see, each key in one program's blocks; a past beyond the table's reach: its last position and the new ones
    for (int i = 0; i < 20000; ++i) {
        const int32_t count = (int32_t)in(0, 90), length = (int32_t)in(0, 400), window = in(0, 1) ? (int32_t)in(1, 200) : 0, past = length - count;
        const int32_t capacity = in(0, 2) ? 1000 : (int32_t)in(0, 400), block = in(0, 1) ? 32 : 64;
        const Sequence q{0, count, length};
        const KeyRange k = tree_range(q, window, capacity);
        const int32_t n = tree_blocks(q, window, block, capacity);
        CHECK(n == 0 || count > 0);
        CHECK(n > 0 || count == 0);
        std::vector<int> taken(401, 0);
        for (int32_t from = 0; from < n;) {
            const int32_t to = (int32_t)in(from + 1, n);
            const KeyRange p = tree_part(k, block, n, from, to);
            if (from) CHECK(p.lo % block == 0);
            for (int j = p.lo; j < p.hi; ++j) ++taken[j];
            CHECK(p.lo >= k.lo && p.hi <= k.hi && (p.hi - 1) / block - p.lo / block < to - from);
            from = to;
        }
        for (int32_t j = 0; j < length && count; ++j) {
            const bool walked = past > capacity ? j >= past - 1 : j >= past || !window || j > past - window;
            CHECK(taken[j] <= 1 && (!walked || taken[j] == 1));
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
def desc(d):
    return d if d is None or isinstance(d, binding.TensorDesc) else binding.make_desc(d)


def ref(d):
    return None if d is None else C.byref(desc(d))


def told(st):
    return binding._STATUS.get(st, st), binding.load().nt_last_error().decode()


def check(call, bad):
    for args, name, text in bad:
        got = call(**args)
        assert got[0] == name and text in got[1], (args, got)


def attended(c=None, q=(5, 4, 64), masks=(5, 1), table=(2, 3), window=0, depths=None, dtype=F16, pm=ADDRESS, pq=ADDRESS):
    c = cache() if c is None else c
    return told(binding.load().nt_sdpa_paged_tree(pq, ref(q), C.byref(c), ADDRESS, ref(table), ADDRESS, ADDRESS, pm, ref(masks), depths, ADDRESS, ref(q), 0.0, window, 0, 0,
                                                  dtype, None))


def test_attention_refusals():
    for over, name, text in BAD_CACHES:
        got = attended(cache(**over))
        assert got[0] == name and text in got[1], (over, got)
    check(attended, [
        (dict(q=(5, 4)), "NT_ERR_SHAPE_MISMATCH", "3-D"),
        (dict(q=(5, 3, 64)), "NT_ERR_SHAPE_MISMATCH", "multiple of the cache's heads"),
        (dict(masks=None), "NT_ERR_INVALID_ARG", "null tensor descriptor"),
        (dict(masks=(5,)), "NT_ERR_SHAPE_MISMATCH", "2-D"),
        (dict(masks=(4, 1)), "NT_ERR_SHAPE_MISMATCH", "differ in tokens"),
        (dict(masks=(5, 0)), "NT_ERR_UNSUPPORTED", "words"),
        (dict(masks=binding.make_desc((5, 2), (4, 2))), "NT_ERR_UNSUPPORTED", "unit stride"),
        (dict(window=-1), "NT_ERR_INVALID_ARG", "negative"),
        (dict(window=9), "NT_ERR_INVALID_ARG", "depths"),
        (dict(dtype=F32), "NT_ERR_UNSUPPORTED", "dtype"),
        (dict(pm=None), "NT_ERR_INVALID_ARG", "null device pointer"),
        (dict(pq=None), "NT_ERR_INVALID_ARG", "null device pointer")])
    assert attended(q=(0, 4, 64), masks=(0, 1), pq=None, pm=None)[0] == 0
    assert attended(table=(0, 3))[0] == 0


def fitted(B=3, table=(3, 5), page=16, capacity=20, tokens=7, **over):
    names = ("lengths", "counts", "pt", "held", "free", "count", "starts", "after", "slots", "positions")
    a = {n: over.get(n, ADDRESS) for n in names}
    return told(binding.load().nt_cache_fit(a["lengths"], a["counts"], B, page, a["pt"], ref(table), a["held"], a["free"], capacity, a["count"], a["starts"], a["after"],
                                            a["slots"], a["positions"], tokens, None))


def test_fit_refusals():
    check(fitted, [
        (dict(table=None), "NT_ERR_INVALID_ARG", "null tensor descriptor"),
        (dict(table=(3, 5, 1)), "NT_ERR_SHAPE_MISMATCH", "2-D"),
        (dict(B=2), "NT_ERR_SHAPE_MISMATCH", "differ in sequences"),
        (dict(B=-1), "NT_ERR_INVALID_ARG", "negative"),
        (dict(capacity=-1), "NT_ERR_INVALID_ARG", "negative"),
        (dict(tokens=-1), "NT_ERR_INVALID_ARG", "negative"),
        (dict(table=binding.make_desc((3, 5), (10, 2))), "NT_ERR_UNSUPPORTED", "unit stride"),
        (dict(page=0), "NT_ERR_UNSUPPORTED", "page_size"),
        (dict(page=(1 << 24) + 1), "NT_ERR_UNSUPPORTED", "page_size"),
        (dict(B=(1 << 24) + 1, table=((1 << 24) + 1, 5)), "NT_ERR_UNSUPPORTED", "too large"),
        (dict(capacity=1 << 31), "NT_ERR_UNSUPPORTED", "pages"),
        (dict(tokens=1 << 31), "NT_ERR_UNSUPPORTED", "tokens")] +
        [({n: None}, "NT_ERR_INVALID_ARG", "null device pointer") for n in ("lengths", "counts", "pt", "held", "free", "count", "starts", "after", "slots", "positions")])


def masked(masks=(5, 1), B=2, window=0, parents=ADDRESS, starts=ADDRESS, pm=ADDRESS, depths=ADDRESS, lengths=None, positions=None):
    return told(binding.load().nt_tree_masks(parents, starts, B, pm, ref(masks), depths, lengths, positions, window, None))


def test_masks_refusals():
    check(masked, [
        (dict(masks=None), "NT_ERR_INVALID_ARG", "null tensor descriptor"),
        (dict(masks=(5,)), "NT_ERR_SHAPE_MISMATCH", "2-D"),
        (dict(masks=(5, 0)), "NT_ERR_UNSUPPORTED", "words"),
        (dict(masks=binding.make_desc((5, 2), (4, 2))), "NT_ERR_UNSUPPORTED", "unit stride"),
        (dict(B=-1), "NT_ERR_INVALID_ARG", "negative"),
        (dict(window=-1), "NT_ERR_INVALID_ARG", "negative"),
        (dict(B=1 << 24), "NT_ERR_UNSUPPORTED", "too many"),
        (dict(lengths=ADDRESS), "NT_ERR_INVALID_ARG", "lengths"),
        (dict(positions=ADDRESS), "NT_ERR_INVALID_ARG", "lengths")] +
        [({n: None}, "NT_ERR_INVALID_ARG", "null device pointer") for n in ("parents", "starts", "pm", "depths")])
    assert masked(masks=(0, 1), parents=None, pm=None)[0] == 0
    assert masked(B=0, starts=None)[0] == 0


def verified(target=(5, 100), draft=(5, 100), path=(2, 4), B=2, dtype=F32, pd=ADDRESS, **over):
    a = {n: over.get(n, ADDRESS) for n in ("target", "ids", "parents", "starts", "uniform", "last", "path", "accepted", "next", "lengths", "after")}
    a["target"] = over.get("pt", ADDRESS)
    a["path"] = over.get("pp", ADDRESS)
    return told(binding.load().nt_verify_tree(a["target"], ref(target), pd, ref(draft), a["ids"], a["parents"], a["starts"], B, a["uniform"], a["last"], a["path"], ref(path),
                                              a["accepted"], a["next"], a["lengths"], a["after"], dtype, None))


def test_verify_refusals():
    check(verified, [
        (dict(dtype=I8), "NT_ERR_UNSUPPORTED", "dtype"),
        (dict(target=None), "NT_ERR_INVALID_ARG", "null tensor descriptor"),
        (dict(draft=None), "NT_ERR_INVALID_ARG", "null tensor descriptor"),
        (dict(path=None), "NT_ERR_INVALID_ARG", "null tensor descriptor"),
        (dict(target=(5,)), "NT_ERR_SHAPE_MISMATCH", "2-D"),
        (dict(draft=(5, 99)), "NT_ERR_SHAPE_MISMATCH", "differ in size"),
        (dict(draft=(4, 100)), "NT_ERR_SHAPE_MISMATCH", "differ in size"),
        (dict(path=(3, 4)), "NT_ERR_SHAPE_MISMATCH", "differ in sequences"),
        (dict(path=(2, 0)), "NT_ERR_SHAPE_MISMATCH", "room"),
        (dict(path=(2, 4, 1)), "NT_ERR_SHAPE_MISMATCH", "2-D"),
        (dict(target=binding.make_desc((5, 100), (200, 2))), "NT_ERR_UNSUPPORTED", "unit stride"),
        (dict(draft=binding.make_desc((5, 100), (200, 2))), "NT_ERR_UNSUPPORTED", "unit stride"),
        (dict(path=binding.make_desc((2, 4), (1, 2))), "NT_ERR_UNSUPPORTED", "unit stride"),
        (dict(target=(5, 1 << 31), draft=(5, 1 << 31)), "NT_ERR_UNSUPPORTED", "vocabulary"),
        (dict(B=-1), "NT_ERR_INVALID_ARG", "negative"),
        (dict(after=None), "NT_ERR_INVALID_ARG", "lengths"),
        (dict(lengths=None), "NT_ERR_INVALID_ARG", "lengths")] +
        [({n: None}, "NT_ERR_INVALID_ARG", "null device pointer") for n in ("pt", "ids", "parents", "starts", "uniform", "last", "pp", "accepted", "next")])
    assert verified(B=0, path=(0, 4), starts=None, pp=None)[0] == 0


def compacted(caches, table=(2, 3), path=(2, 4), n=None, **over):
    a = {n: over.get(n, ADDRESS) for n in ("pt", "lengths", "pp", "accepted")}
    array = None if caches is None else (binding.PagedCache * max(1, len(caches)))(*caches)
    return told(binding.load().nt_cache_compact(array, len(caches or ()) if n is None else n, a["pt"], ref(table), a["lengths"], a["pp"], ref(path), a["accepted"], None))


def test_compact_refusals():
    for over, name, text in BAD_CACHES:
        if "the tokens' type" in text and over["dtype"] == BF16:
            continue                                                       # (a cache of the other 16-bit type is as good here)
        got = compacted([cache(), cache(**over)])
        assert got[0] in (name, "NT_ERR_SHAPE_MISMATCH", "NT_ERR_UNSUPPORTED"), (over, got)
    other = binding.make_desc((4, 16, 2, 64), (2 * 16 * 2 * 64, 2 * 64, 64, 1))
    check(compacted, [
        (dict(caches=None, n=1), "NT_ERR_INVALID_ARG", "null cache"),
        (dict(caches=[], n=-1), "NT_ERR_INVALID_ARG", "negative"),
        (dict(caches=[cache(), cache(dtype=BF16)]), "NT_ERR_SHAPE_MISMATCH", "one type"),
        (dict(caches=[cache(), cache(pages=5)]), "NT_ERR_SHAPE_MISMATCH", "one layout"),
        (dict(caches=[cache(), cache(dv=other)]), "NT_ERR_SHAPE_MISMATCH", "one layout"),
        (dict(caches=[cache(dtype=F32)]), "NT_ERR_UNSUPPORTED", "dtype"),
        (dict(caches=[cache(dtype=E4M3)]), "NT_ERR_INVALID_ARG", "needs scales"),
        (dict(caches=[cache(), cache(k=ADDRESS + 4096)]), "NT_ERR_INVALID_ARG", "listed twice"),
        (dict(caches=[cache(), cache()]), "NT_ERR_INVALID_ARG", "listed twice"),
        (dict(caches=[cache()], table=(1 << 23, 3), path=(1 << 23, 4)), "NT_ERR_UNSUPPORTED", "one launch"),
        (dict(caches=[cache()], table=None), "NT_ERR_INVALID_ARG", "null tensor descriptor"),
        (dict(caches=[cache()], table=(2, 3, 1)), "NT_ERR_SHAPE_MISMATCH", "2-D"),
        (dict(caches=[cache()], path=(3, 4)), "NT_ERR_SHAPE_MISMATCH", "differ in sequences"),
        (dict(caches=[cache()], path=binding.make_desc((2, 4), (1, 2))), "NT_ERR_UNSUPPORTED", "unit stride"),
        (dict(caches=[cache()], table=binding.make_desc((2, 3), (1, 2))), "NT_ERR_UNSUPPORTED", "unit stride"),
        (dict(caches=[cache()], table=(1 << 30, 3), path=(1 << 30, 4)), "NT_ERR_UNSUPPORTED", "too large")] +
        [(dict(caches=[cache()], **{n: None}), "NT_ERR_INVALID_ARG", "null device pointer") for n in ("pt", "lengths", "pp", "accepted")])
    assert compacted([])[0] == 0
    assert compacted([cache()], table=(0, 3), path=(0, 4))[0] == 0


def test_tensors_off_the_gpu_are_refused():
    f, i, j = torch.zeros(3, 2, 64, dtype=torch.float16), torch.zeros(4, dtype=torch.int32), torch.zeros(3, 1, dtype=torch.int64)
    c, table = torch.zeros(4, 16, 2, 64, dtype=torch.float16), torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(ValueError):
        nt.sdpa_paged_tree(f, c, c, table, i[:2], i[:1], j, torch.empty_like(f))
    with pytest.raises(ValueError):
        nt.cache_fit(i[:1], i[:1], 16, table, i[:1], i, i[:1], i[:2], i[:1], j[:, 0], i[:3])
    with pytest.raises(ValueError):
        nt.tree_masks(i[:3], i[:2], j, i[:3])
    with pytest.raises(ValueError):
        nt.verify_tree(torch.zeros(3, 9), None, j[:, 0], i[:3], i[:2], torch.zeros(3), torch.zeros(1), table, i[:1], j[:1, 0])
    with pytest.raises(ValueError):
        nt.cache_compact([(c, c)], table, i[:1], table, i[:1])
