"""Page selection over more pages than are ranked on chip (4096), against its definition."""
import numpy as np
import pytest
import torch

import paper_2011_09398_amd as lce
from tests.kv4_util import PAGE

pytestmark = pytest.mark.gpu


def best_pages(score, count, first, last):
    n = len(score)
    page = np.arange(n)
    rank = np.where((page < first) | (page >= n - last), 10 ** 6, score)
    chosen = np.sort(np.lexsort((page, -rank))[:count])
    return np.concatenate((chosen, np.full(count - len(chosen), -1)))


@pytest.mark.parametrize("width", [4095, 4096, 4097, 9001])
@pytest.mark.parametrize("chunk", [0, 100, 10 ** 6])
@pytest.mark.parametrize("heads,kv_heads", [(2, 1), (6, 2)])
def test_select_of_more_pages_than_are_held(width, chunk, heads, kv_heads):
    """A few pages of memory, many times in the tables; two sequences, split or not, and one
    workspace for calls with other queries, so that a rank left over would show."""
    dim, pages, seqs = 64, 50, 2
    rng = np.random.default_rng(width)
    data = rng.integers(0, 256, (pages, kv_heads, 76 * dim)).astype(np.uint8)
    table = rng.integers(0, pages, (seqs, width)).astype(np.int32)
    lengths = np.array([width * PAGE - 13, (width - 3) * PAGE], np.int32)
    bits = np.unpackbits(data[:, :, 68 * dim:].reshape(pages, kv_heads, PAGE, dim // 8), axis=-1,
                         bitorder="little")
    sign = 1 - 2 * bits.astype(np.int64)                # [pages, kv_heads, 64, dim]
    cache = lce.KV4Cache(kv_heads, dim, data=torch.from_numpy(data).cuda())
    dev = (torch.from_numpy(table).cuda(), torch.arange(seqs + 1, dtype=torch.int32).cuda(),
           torch.from_numpy(lengths).cuda())
    ws = lce.kv4_workspace(cache, torch.zeros(seqs, heads, dim, device="cuda").half(), dev[0])
    with lce.tuning(kv4_chunk=chunk):
        for count, first, last in ((5, 1, 1), (width - 2, 0, 0), (4500, 3, 2), (64, 0, 0), (64, 1, 1)):
            q = torch.from_numpy(rng.standard_normal((seqs, heads, dim))).half()
            got = lce.kv4_select(cache, q.cuda(), *dev, count, keep_first=first, keep_last=last,
                                 workspace=ws).cpu().numpy()
            assert not ws[:lce.KV4_WORKSPACE_ZERO].any()
            total = np.where(q.numpy() < 0, -1, 1).reshape(seqs, kv_heads, -1, dim).sum(2)
            for b in range(seqs):
                for h in range(kv_heads):
                    score = sign[:, h] @ total[b, h].astype(np.int64)       # [pages, 64]
                    mine = score.max(-1)[table[b, :-(-lengths[b] // PAGE)]]
                    over = -lengths[b] % PAGE
                    if over:
                        mine[-1] = score[table[b, len(mine) - 1], :PAGE - over].max()
                    assert np.array_equal(got[b, h], best_pages(mine, count, first, last)), (b, h, count)
