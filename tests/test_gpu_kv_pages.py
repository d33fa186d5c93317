"""Pages of the 4-bit cache when a table holds ids that do not exist: what cannot be served changes nothing and says so."""
import numpy as np
import pytest
import torch

import gpu_util as G
from paper_2310_08041_b200 import binding as B
from test_gpu_kv import ints, pool_state, random_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [20, -5, 2 ** 31 - 1, -1])
@pytest.mark.parametrize("at", ["first", "full", "last"])
def test_forking_a_sequence_with_a_page_that_does_not_exist(at, bad):
    """Of five entries, two have a parent with a bad page (a full one, or the partly filled last): their children stay unused, no count
    and no page changes for them, and the pages they would have copied into go to the others."""
    pages, seqs, width, page = 20, 8, 6, 16
    cache, pool = random_cache(81, 2, pages, 2, page, 64), B.KvPool.empty(pages, seqs, width)
    B.qllm_kv_pages_extend(cache, pool, ints([70, 70, 33, 0, 0, 0, 0, 0]))
    place = {"first": 0, "full": 3, "last": 4}[at]
    lost = int(pool.table[1, place])
    pool.table[1, place] = bad
    B.qllm_poll_status()
    arrays = (cache.k_codes, cache.k_param, cache.v_codes, cache.v_param)
    before, refs0, table0 = [t.clone() for t in arrays], pool.refs.tolist(), pool.table.tolist()
    fresh = B.qllm_kv_pages_fork(cache, pool, ints([1, 0, 1, 2, 0]), ints([3, 4, 5, 6, 7])).tolist()
    assert B.qllm_poll_status() == B.QLLM_ERR_PAGE
    free = [p for p in range(pages) if refs0[p] == 0]
    assert fresh == [-2, free[0], -2, free[1], free[2]]
    refs, table, lens = (a.tolist() for a in pool_state(pool))
    assert lens == [70, 70, 33, 0, 70, 0, 33, 70]
    assert table[:4] == table0[:4] and table[5] == table0[5]
    assert table[4] == table0[0][:4] + [free[0], -1] and table[7] == table0[0][:4] + [free[2], -1]
    assert table[6] == table0[2][:2] + [free[1], -1, -1, -1]
    want = list(refs0)
    for p in table[4] + table[6] + table[7]:
        if p >= 0:
            want[p] += 1
    assert refs == want and want[lost] == 1
    for t, old in zip(arrays, before):
        old[:, free[0]], old[:, free[1]], old[:, free[2]] = old[:, table0[0][4]], old[:, table0[2][2]], old[:, table0[0][4]]
        assert torch.equal(t, old)


def test_a_bad_page_behind_a_parents_length_does_not_matter():
    cache, pool = random_cache(82, 1, 9, 1, 16, 64), B.KvPool.empty(9, 3, 4)
    B.qllm_kv_pages_extend(cache, pool, ints([32, 0, 0]))
    pool.table[0, 2] = 99                                    # the length ends in front of it
    B.qllm_poll_status()
    assert B.qllm_kv_pages_fork(cache, pool, ints([0]), ints([2])).tolist() == [-1]
    assert B.qllm_poll_status() == B.QLLM_OK and pool.table[2].tolist() == [0, 1, -1, -1]


@pytest.mark.parametrize("seed", range(4))
def test_many_entries_with_bad_pages_among_their_parents(seed):
    """More entries than a CTA has warps, against the rules applied one entry after the other."""
    rng = np.random.RandomState(seed)
    pages, seqs, width, page = 4000, 400, 12, 16
    cache, pool = random_cache(83, 1, pages, 1, page, 64), B.KvPool.empty(pages, seqs, width)
    lens = np.where(np.arange(seqs) < 90, rng.randint(0, width * page + 1, seqs), 0)
    B.qllm_kv_pages_extend(cache, pool, ints(lens))
    assert B.qllm_poll_status() == B.QLLM_OK
    table = pool.table.cpu().numpy()
    bad = set()
    for s in rng.choice(90, 30, replace=False):
        used = -(-lens[s] // page)
        if used:
            table[s, rng.randint(used)] = rng.choice([pages, -7, -1, 10 ** 9])
            bad.add(int(s))
    pool.table.copy_(torch.from_numpy(table))
    refs = pool.refs.cpu().numpy().copy()
    parent, child = rng.randint(0, 90, 300), 90 + rng.permutation(300)
    fresh = B.qllm_kv_pages_fork(cache, pool, ints(parent), ints(child)).tolist()
    assert B.qllm_poll_status() == B.QLLM_ERR_PAGE
    free, want = [p for p in range(pages) if refs[p] == 0], []
    new_lens = lens.copy()
    for a, c in zip(parent, child):
        if int(a) in bad:
            want.append(-2)
            continue
        full, rest = divmod(int(lens[a]), page)
        table[c, :full] = table[a, :full]
        refs[table[a, :full]] += 1
        want.append(-1)
        if rest:
            want[-1] = free.pop(0)
            table[c, full] = want[-1]
            refs[want[-1]] = 1
        new_lens[c] = lens[a]
    got = pool_state(pool)
    assert fresh == want and np.array_equal(got[0], refs) and np.array_equal(got[1], table) and np.array_equal(got[2], new_lens)
