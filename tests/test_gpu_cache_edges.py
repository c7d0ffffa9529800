"""The paged cache on the GPU where tables, values or sizes are out of the ordinary."""
import pytest
import torch

from paged_reference import Paged

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def attnw():
    from paper_2407_13885_b200 import binding
    yield binding
    assert binding.query_status() == 0


def bits(x):
    return x.view(torch.int32 if x.dtype == torch.float32 else torch.int16).cpu()


# ---- eviction ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_eviction_of_keys_without_a_page(attnw, in_place, d):
    # A page that the cache does not have reads as zeros: a key of it that stays is zero in its new place, whatever was there.
    page, budget, recent = 16, 40, 10
    c = Paged([(0, 100), (0, 130)], 2, d, page, spare=9)
    c.table[0, 3], c.table[0, 6], c.table[1, 2], c.table[1, 8] = -1, c.pages, 2 ** 31 - 1, -5
    mass = torch.rand(2, 2, c.width * page, generator=c.gen).cuda()
    mass[0, :, 48:64] += 1.0                       # the keys of missing pages are among those that stay
    mass[1, 0, 32:48] += 1.0
    K0, V0 = c.K.cpu(), c.V.cpu()
    before = c.table.cpu()
    out = None if in_place else torch.tensor(c.spare[:6], dtype=torch.int32, device="cuda").view(2, 3)
    kept, lengths, _ = attnw.cache_evict(c.K, c.V, c.table, c.lengths, mass, budget, recent, table_out=out)
    assert lengths.tolist() == [40, 40] and torch.equal(c.table.cpu(), before)
    to = (c.table if in_place else out).cpu().long()
    want_K, want_V = K0.clone(), V0.clone()
    zeros = 0
    for b in range(2):
        for h in range(2):
            for t in range(budget):
                s = int(kept[b, h, t])
                source, target = int(before[b, s // page]), int(to[b, t // page])
                if not 0 <= target < c.pages:
                    continue
                there = 0 <= source < c.pages
                zeros += not there
                want_K[target, h, t % page] = K0[source, h, s % page] if there else 0.0
                want_V[target, h, t % page] = V0[source, h, s % page] if there else 0.0
    assert zeros >= 16
    assert torch.equal(bits(c.K), bits(want_K)) and torch.equal(bits(c.V), bits(want_V))
