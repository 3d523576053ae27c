"""What needs no device of the calls around a paged cache: their struct as the header lays it out, and calls without a context."""
import ctypes

from paper_2603_17803_amd import binding


def test_struct_layout_matches_the_header():
    # dtype(4) pad(4) k v (8 each) L P H page d (4 each) pad(4) table len refs (8 each) rows cap (4 each) = 80 bytes on LP64
    c = binding.swarm_cache
    assert [getattr(c, f).offset for f, _ in c._fields_] == [0, 8, 16, 24, 28, 32, 36, 40, 48, 56, 64, 72, 76]
    assert ctypes.sizeof(c) == 80


def test_null_context_is_rejected():
    c = binding.swarm_cache()
    assert binding.swarm_tree_attend(0, c, 0, 0, None, None, 1, 1, 1, None, None, None, 0, 0, 1.0, 0, None) == binding.SWARM_EINVAL
    assert binding.swarm_cache_fork(0, c, 0, None, 0, 0, 0) == binding.SWARM_EINVAL
    assert binding.swarm_cache_append(0, c, 0, 0, 1, 1, None, 1, None, 0) == binding.SWARM_EINVAL
    assert binding.swarm_cache_compact(0, c, 0, 0, 0) == binding.SWARM_EINVAL
    assert binding.swarm_beam_select(0, 0, 0, 8, 0, None, -1, 1, 1, 8, 1, 0, 0, 0, None, None, 0, None) == binding.SWARM_EINVAL


def test_cache_has_its_fields_by_name():
    c = binding.Cache("k", "v", "table", "length")
    assert (c.k, c.v, c.table, c.length, c.refs) == ("k", "v", "table", "length", None)
