"""Forks that copy unequal numbers of pages, and forks whose parents alternate, in calls of up to some
thousand forks: exact, against the plain definition."""
import numpy as np
import pytest
import torch

from paper_2609_31395_amd import actkv
from test_gpu_pages import _fork_reference

pytestmark = pytest.mark.gpu
DEV = "cuda"


def run(forks, parents, stride, P, rows, seed):
    rng = np.random.default_rng(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    kv = torch.randint(-32768, 32767, (2, P, 16, 1, 64), dtype=torch.int16, device=DEV, generator=g)
    bt = np.full((rows, stride), -9, np.int32)
    perm = rng.permutation(P).astype(np.int32)
    for r in range(parents):
        bt[r] = perm[r * stride:(r + 1) * stride]
    bt[0, stride // 3] = -1   # a page outside the pool
    f = actkv.Forks(*np.array(forks, np.int32).T).to_device(DEV)
    free = perm[parents * stride:][:f.num_fresh].copy()
    assert free.size == f.num_fresh   # every fresh page is needed
    refs = rng.integers(0, 3, P).astype(np.int32)
    want = _fork_reference(forks, kv, bt, free, refs)
    bt_d, refs_d = torch.from_numpy(bt).to(DEV), torch.from_numpy(refs).to(DEV)
    actkv.fork_pages(f, kv, bt_d, torch.from_numpy(free).to(DEV), refs_d)
    np.testing.assert_array_equal(bt_d.cpu().numpy(), want[1])
    np.testing.assert_array_equal(refs_d.cpu().numpy(), want[2])
    assert torch.equal(kv, want[0])


@pytest.mark.parametrize("n", [1, 2, 255, 256, 257, 700, 3000])
@pytest.mark.parametrize("long_at", ["first", "last"])
def test_one_fork_copies_its_row_and_the_others_little(n, long_at):
    stride, rng = 300, np.random.default_rng(n)
    forks = [[int(rng.integers(0, 3)), 3 + i, *sorted(rng.integers(0, 4, 2).tolist())] for i in range(n)]
    at = 0 if long_at == "first" else n - 1
    forks[at][2:] = [0, stride]
    run(forks, 3, stride, 3 * stride + 300 + 3 * n, 3 + n, n)


@pytest.mark.parametrize("n", [63, 64, 65, 130, 300])
def test_parents_that_alternate(n):
    """Runs of a parent's forks, cut by other parents' and by the groups of 64 that are counted together."""
    stride, rng = 1100, np.random.default_rng(n)
    parent = {0: lambda i: i % 2, 1: lambda i: i // 3 % 3, 2: lambda i: int(rng.integers(0, 3))}[n % 3]
    forks = []
    for i in range(n):
        shared = int(rng.choice([0, 5, 1024, 1025, stride]))
        forks.append([parent(i), 3 + i, shared, min(stride, shared + int(rng.integers(0, 3)))])
    run(forks, 3, stride, 3 * stride + 3 * n, 3 + n, n)


def test_no_fork_changes_nothing():
    kv = torch.zeros(2, 6, 16, 1, 64, dtype=torch.int16, device=DEV)
    bt = torch.full((3, 2), 5, dtype=torch.int32, device=DEV)
    refs = torch.ones(6, dtype=torch.int32, device=DEV)
    f = actkv.Forks.of_lengths([], [], np.zeros((0, 1)))
    actkv.fork_pages(f, kv, bt, None, refs)
    actkv.fork_pages(f.to_device(DEV), kv, bt, None, refs)
    assert (bt == 5).all() and (refs == 1).all() and (kv == 0).all()


@pytest.mark.parametrize("n,copied_by", [(64, 64), (65, 65), (128, 1), (4096, 4096), (4097, 4097), (4160, 30), (8193, 8193),
                                         (9000, 3)])
def test_forks_past_what_is_added_up_at_a_time(n, copied_by):
    """The last `copied_by` forks copy up to three pages each, the others none."""
    rng = np.random.default_rng(n)
    forks = [[int(rng.integers(0, 3)), 3 + i, 2, 2 if i < n - copied_by else 2 + int(rng.integers(0, 4))] for i in range(n)]
    forks[-1][3] = 5   # the last page of all is the last fork's
    run(forks, 3, 6, 18 + 3 * n, 3 + n, n)
