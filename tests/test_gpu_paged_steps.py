"""PagedLatentCache on the GPU: compaction that moves pages, a device named without its index, and the
tokens after them against the float64 oracle (tolerance: tests/test_gpu_paged.py)."""
import pytest

from paper_2607_27269_amd import configs
from test_gpu_paged_cache import Model

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,ps", [("05b", 16), ("1b", 7)])
def test_compaction_moves_pages_and_keeps_the_tokens(name, ps):
    print(f"[paged] compaction {name}, pages of {ps}", flush=True)
    m = Model(name, n_pages=60, ps=ps, seed=100 + ps)
    first, b, c = m.add(), m.add(), m.add()
    m.step([first], [5 * ps + 3])            # the lowest pages
    m.step([b, c], [3 * ps + 1, 2 * ps])
    d = m.fork(b)
    m.cache.free(first)
    used = len({p for pages in m.cache.alloc.pages.values() for p in pages})
    assert max(p for pages in m.cache.alloc.pages.values() for p in pages) >= used
    assert m.cache.compact() == used         # six low pages free, every page in use behind them or moved
    assert max(p for pages in m.cache.alloc.pages.values() for p in pages) == used - 1
    # whatever lies behind the pages in use is free
    m.cache.pool[:, used:] = float("nan")
    m.step([b, c, d], [1, 1, 1])
    m.step([d, b], [2, ps])


def test_the_device_keeps_its_index():
    import torch
    from paper_2607_27269_amd.paged import PagedLatentCache
    c = PagedLatentCache(configs.get(1), 1, 4, 16, device="cuda")
    assert c.device == c.pool.device and c.device.index == torch.cuda.current_device()
