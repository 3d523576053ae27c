"""Arguments of the calls around a paged cache that the binding refuses, without a device: the library's calls are not reached."""
import pytest

torch = pytest.importorskip("torch")

from paper_2603_17803_amd import binding  # noqa: E402


@pytest.fixture
def host(monkeypatch):
    """The binding's checks on tensors of the host, and calls that only count."""
    s = object.__new__(binding.Swarm)
    s.torch, s.device, s.ctx = torch, torch.device("cpu"), None
    s._index, s._i32, s._f32 = torch.empty(1).get_device(), torch.int32, torch.float32
    s._kinds = {torch.bfloat16: binding.SWARM_BF16, torch.float16: binding.SWARM_FP16, torch.float32: binding.SWARM_FP32}
    s.reached = []
    for name in ("swarm_tree_attend", "swarm_cache_append", "swarm_cache_fork", "swarm_cache_compact", "swarm_beam_select"):
        monkeypatch.setattr(binding, name, lambda *a, name=name: s.reached.append(name) or binding.SWARM_OK)
    return s


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def cache():
    pool = torch.zeros((1, 4, 2, 4, 32), dtype=torch.bfloat16)
    return binding.Cache(pool, pool.clone(), i32(2, 3), i32(2), i32(4))


def test_the_calls_are_reached(host):
    q, new = torch.zeros((2, 3, 4, 32), dtype=torch.bfloat16), torch.zeros((1, 2, 3, 2, 32), dtype=torch.bfloat16)
    host.tree_attend(cache(), 0, q, new[0], new[0], sel=i32(2, 2, 1))
    host.cache_append(cache(), new, new, path=i32(2, 1))
    host.beam_select(torch.zeros((2, 3, 5)), torch.zeros((2, 3)), 2)
    assert host.reached == ["swarm_tree_attend", "swarm_cache_append", "swarm_beam_select"]


def test_an_empty_selection_is_not_the_whole_context(host):
    q = torch.zeros((2, 1, 4, 32), dtype=torch.bfloat16)
    for unit in ("page", "token"):
        with pytest.raises(ValueError):
            host.tree_attend(cache(), 0, q, sel=i32(2, 2, 0), unit=unit)
    assert not host.reached


def test_an_empty_path_is_not_all_tokens(host):
    new = torch.zeros((1, 2, 3, 2, 32), dtype=torch.bfloat16)
    for n in (None, i32(2)):
        with pytest.raises(ValueError):
            host.cache_append(cache(), new, new, n=n, path=i32(2, 0))
    assert not host.reached


def test_no_optional_tensor_without_elements_counts_as_absent(host):
    """The address of a tensor without elements is NULL, which the library takes for an argument that is not there."""
    q = torch.zeros((2, 0, 4, 32), dtype=torch.bfloat16)
    none = torch.zeros((2, 0, 2, 32), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        host.tree_attend(cache(), 0, q, none, none)
    with pytest.raises(ValueError):
        host.beam_select(torch.zeros((2, 3, 5)), torch.zeros((2, 3)), 2, hist=i32(2, 3, 0), step=i32(1), hist_out=i32(2, 2, 0))
    with pytest.raises(ValueError):
        host.beam_select(torch.zeros((2, 0, 5)), torch.zeros((2, 0)), 2, finished=torch.zeros((2, 0), dtype=torch.uint8), eos=1)
    assert not host.reached
