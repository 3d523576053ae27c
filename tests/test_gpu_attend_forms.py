"""Attention over a paged cache at either side of the sizes that decide how a pair's parts are finished, and long chains of tokens."""
import pytest

from test_gpu_attend import Problem

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def sw():
    from paper_2603_17803_amd import binding
    s = binding.Swarm(0)
    yield s
    assert s.device_status() == 0
    s.close()


# workgroups of 16 rows of a pair: 512, 504, 256, 128, 144, 128, 120; parts of a pair at most: 8, 8, 16, 3, 3, 4, 5
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("B,H,T,G,n", [(8, 8, 32, 4, 1024), (9, 8, 28, 4, 900), (4, 8, 32, 4, 2048), (2, 8, 32, 4, 300), (2, 8, 33, 4, 300), (16, 8, 4, 4, 600), (15, 8, 4, 4, 700)])
def test_pairs_that_few_and_many_waves_finish(sw, dtype, B, H, T, G, n):
    Problem(B + T, dtype, B, T, H, G, 32, 16, [n - 7 * b for b in range(B)], tree=True, n_new=[T] * (B - 1) + [T - 1]).check(sw)


@pytest.mark.parametrize("T,G,d", [(128, 2, 64), (129, 1, 64), (200, 2, 64), (256, 1, 64), (255, 4, 32), (130, 1, 160)])
def test_long_chains(sw, T, G, d):
    """More than 100 tokens without a mask: a piece of a prompt."""
    Problem(T + d, "bf16" if T % 2 else "fp16", 3, T, 1, G, d, 16, [200, 0, 33], n_new=[T, T - 1, T // 2]).check(sw)
