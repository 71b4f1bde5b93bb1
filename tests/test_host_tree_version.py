"""The version that tells the interface with drafted trees from the one without."""

import re

import paper_2507_11978_amd as nt


def test_the_version_is_not_that_of_the_library_without_trees():
    assert tuple(int(n) for n in re.match(r"nt-mi355x (\d+)\.(\d+) \(gfx950\)$", nt.version()).groups()) >= (0, 9)
    for name in ("cache_fit", "tree_masks", "sdpa_paged_tree", "verify_tree", "cache_compact"):
        assert callable(getattr(nt, name)) and hasattr(nt.load(), "nt_" + name)
