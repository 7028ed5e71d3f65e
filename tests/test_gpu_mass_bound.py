"""The bound that a call for the mass of many rows is given: sequences of exactly so many tokens and of one more, and those that hold more tokens but need no
more slots, in each of the three ways that the sums over rows take."""
import numpy as np
import pytest
import torch

import paper_2510_05373_amd as kv
from tests.kvlinc_testlib import to_dev
from tests.test_gpu_mass import check_all, prepared, prior_of

pytestmark = pytest.mark.gpu


# 16, 600 and 1200 rows a KV head: one launch, two, three
@pytest.mark.parametrize("T", [4, 150, 300])
@pytest.mark.parametrize("bound, lengths, room", [(300, [300, 301, 512, 513, 129, 0], 0), (1, [1, 2, 128, 129, 256, 257], 0), (384, [384, 385, 512, 383], 0),
                                                  (383, [384, 383], 256), (300, [512], 0)])
def test_sequences_around_the_bound(bound, lengths, room, T):
    rows = [min(T, max(n, 1)) for n in lengths]
    cache, K, V, q, nq = prepared(1800 + bound, 8, 2, lengths, T, room=room)
    mass = prior_of(cache)
    out = torch.full_like(mass, 7.0)
    n_rows = to_dev(np.asarray(rows, np.int32))
    cache.attention_mass(to_dev(q), mass, n_rows=n_rows, decay=0.5, mass_out=out, max_context=bound)
    assert cache.status.item() == kv.KVLINC_ST_BOUND and int(cache.split_done.abs().sum()) == 0
    # a sequence of more tokens keeps what it had, faded; the others' rows count
    check_all(cache, K, V, q, nq, [r if n <= bound else 0 for r, n in zip(rows, lengths)], out, mass, 0.5, 2)


@pytest.mark.parametrize("T", [4, 150, 300])
@pytest.mark.parametrize("bound", [384, 385, 0, -5, 1 << 30])
def test_a_bound_that_holds_reports_nothing(bound, T):
    lengths = [384, 300, 1, 0]  # (the first fills its cache)
    rows = [min(T, max(n, 1)) for n in lengths]
    cache, K, V, q, nq = prepared(1850, 8, 2, lengths, T, room=256)
    out = torch.full_like(cache.new_mass(), 7.0)
    cache.attention_mass(to_dev(q), None, n_rows=to_dev(np.asarray(rows, np.int32)), mass_out=out, max_context=bound)
    assert cache.status.item() == 0
    check_all(cache, K, V, q, nq, rows, out, None, 1.0, 2)
