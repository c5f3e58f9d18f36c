"""Forks and shared pages (actkv_fork_pages, actkv_acquire_pages, actkv_release_pages): whole numbers
and copies, compared exactly with the plain definition."""
import numpy as np
import pytest
import torch

from paper_2609_31395_amd import actkv

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    actkv.load_library()


def _release_reference(pages, refs):
    refs = refs.copy()
    for p in pages.reshape(-1):
        if 0 <= p < refs.size:
            refs[p] = max(int(refs[p]) - 1, 0) if refs[p] > 0 else refs[p]
    return refs


@pytest.mark.parametrize("n,num_pages", [(0, 10), (1, 1), (5, 33), (300, 100), (1023, 5000), (1024, 256), (1025, 257),
                                         (5000, 8192), (20000, 70001), (3000, 1_200_000), (2000, 4_300_000)])
def test_release_lists_the_pages_that_nobody_holds(n, num_pages):
    rng = np.random.default_rng(n)
    refs = rng.integers(0, 4, num_pages).astype(np.int32)
    pages = rng.integers(-2, num_pages + 2, n).astype(np.int32)
    pages[rng.random(n) < 0.1] = -(1 << 31)
    refs_d, pages_d = torch.from_numpy(refs).to(DEV), torch.from_numpy(pages).to(DEV)
    for _ in range(3):
        want = _release_reference(pages, refs)
        gone = np.nonzero((refs > 0) & (want == 0))[0]
        freed, count = actkv.release_pages(pages_d, refs_d)
        assert int(count) == gone.size
        np.testing.assert_array_equal(freed.cpu().numpy(), np.concatenate([gone, np.full(n - gone.size, -1)]))
        np.testing.assert_array_equal(refs_d.cpu().numpy(), want)
        refs = want


@pytest.mark.parametrize("rows,row_len", [(1, 1500), (20, 100), (64, 40), (9, 257), (17, 2188), (2000, 1), (100, 2188)])
def test_release_of_rows_that_share_pages(rows, row_len):
    """Runs of rows with the same pages in the same places, cut by others, longer and shorter than
    what a thread takes."""
    rng = np.random.default_rng(rows)
    num_pages = 5000
    base = rng.integers(-1, num_pages, (rows, row_len)).astype(np.int32)
    owner = np.sort(rng.integers(0, max(1, rows // 3), rows))
    pages = base[owner]
    pages[rng.random(pages.shape) < 0.02] = -1
    refs = rng.integers(0, 8, num_pages).astype(np.int32)
    refs_d, pages_d = torch.from_numpy(refs).to(DEV), torch.from_numpy(pages).to(DEV)
    for _ in range(2):
        want = _release_reference(pages, refs)
        gone = np.nonzero((refs > 0) & (want == 0))[0]
        freed, count = actkv.release_pages(pages_d, refs_d)
        assert int(count) == gone.size
        np.testing.assert_array_equal(freed.cpu().numpy()[:gone.size], gone)
        assert (freed[gone.size:] == -1).all()
        np.testing.assert_array_equal(refs_d.cpu().numpy(), want)
        refs = want


def test_acquire_counts_every_entry():
    pages = torch.tensor([3, 3, -1, 9, 10, 0, 3, -(1 << 31), 1 << 30], dtype=torch.int32, device=DEV)
    refs = torch.zeros(10, dtype=torch.int32, device=DEV)
    actkv.acquire_pages(pages, refs)
    assert refs.tolist() == [1, 0, 0, 3, 0, 0, 0, 0, 0, 1]
    freed, count = actkv.release_pages(pages, refs)
    assert refs.tolist() == [0] * 10 and int(count) == 3 and freed.tolist() == [0, 3, 9] + [-1] * 6
    actkv.acquire_pages(torch.empty(0, dtype=torch.int32, device=DEV), refs)


def _fork_reference(forks, kv, bt, free, refs):
    kv, bt, refs, at = kv.clone(), bt.copy(), refs.copy(), 0
    src_bt = bt.copy()
    P = kv.shape[1]
    src = kv.clone()
    for parent, child, shared, pages in forks:
        row = np.full(bt.shape[1], -1, np.int32)
        row[:shared] = src_bt[parent, :shared]
        for p in row[:shared]:
            if 0 <= p < P:
                refs[p] += 1
        for i in range(shared, pages):
            f, s = free[at], src_bt[parent, i]
            at += 1
            row[i] = f
            if 0 <= f < P:
                refs[f] = 1
                if 0 <= s < P:
                    kv[:, f] = src[:, s]
        bt[child] = row
    return kv, bt, refs


@pytest.mark.parametrize("heads,dim", [(1, 64), (3, 64), (4, 128), (8, 128)])
@pytest.mark.parametrize("stride", [1, 40, 1500])
def test_fork_shares_full_pages_and_copies_the_others(heads, dim, stride):
    rng = np.random.default_rng(stride + heads)
    P, rows = 4000, 12
    g = torch.Generator(device=DEV).manual_seed(stride)
    kv = torch.randint(-32768, 32767, (2, P, 16, heads, dim), dtype=torch.int16, device=DEV, generator=g)
    bt = np.full((rows, stride), -9, np.int32)
    perm = rng.permutation(P).astype(np.int32)
    bt[0], bt[1] = perm[:stride], perm[stride:2 * stride]
    bt[2] = bt[0]
    bt[2, stride // 2] = -1          # a page outside the pool
    free = perm[2 * stride:].copy()
    m = min(stride, 40)
    forks = np.array([[0, 5, stride, stride], [0, 6, stride - min(1, stride), stride], [1, 3, 0, m],
                      [2, 11, max(0, stride - m), stride], [1, 4, 0, 0], [2, 7, stride // 2, stride // 2]])
    # several forks of one parent in a row, sharing different numbers of pages
    more = [[1, 8, stride, stride], [1, 9, m, m], [1, 10, stride, stride]]
    forks = np.concatenate([forks, more])
    f = actkv.Forks(*forks.T).to_device(DEV)
    refs = rng.integers(0, 3, P).astype(np.int32)
    want = _fork_reference(forks, kv, bt, free, refs)
    bt_d, refs_d = torch.from_numpy(bt).to(DEV), torch.from_numpy(refs).to(DEV)
    free_d = torch.from_numpy(free).to(DEV)
    actkv.fork_pages(f, kv, bt_d, free_d, refs_d)
    np.testing.assert_array_equal(bt_d.cpu().numpy(), want[1])
    np.testing.assert_array_equal(refs_d.cpu().numpy(), want[2])
    assert torch.equal(kv, want[0])


def test_fork_without_counts_and_with_fresh_pages_outside_the_pool():
    kv = torch.randint(-99, 99, (2, 6, 16, 2, 64), dtype=torch.int16, device=DEV)
    before = kv.clone()
    bt = torch.tensor([[1, 2], [-5, -5], [-5, -5]], dtype=torch.int32, device=DEV)
    f = actkv.Forks([0, 0], [1, 2], [1, 0], [2, 2]).to_device(DEV)
    free = torch.tensor([6, 4, -1], dtype=torch.int32, device=DEV)
    actkv.fork_pages(f, kv, bt, free)
    assert bt.tolist() == [[1, 2], [1, 6], [4, -1]]
    assert torch.equal(kv[:, 4], before[:, 1])
    kv[:, 4] = before[:, 4]
    assert torch.equal(kv, before)


def test_forks_of_lengths():
    f = actkv.Forks.of_lengths([0, 1], [2, 3], [[33, 16], [0, 5]])
    assert f.shared.tolist() == [1, 0] and f.pages.tolist() == [3, 1] and f.num_fresh == 3
    f = actkv.Forks.of_lengths([0], [1], [[32, 48]], share=False)
    assert f.shared.tolist() == [0] and f.pages.tolist() == [3]


def test_fork_and_release_replayed_from_a_graph():
    rng = np.random.default_rng(5)
    P, W = 3000, 200
    kv = torch.randint(-99, 99, (2, P, 16, 2, 64), dtype=torch.int16, device=DEV)
    perm = torch.from_numpy(rng.permutation(P).astype(np.int32)).to(DEV)
    bt = torch.full((6, W), -1, dtype=torch.int32, device=DEV)
    bt[0], bt[1] = perm[:W], perm[W:2 * W]
    refs = torch.zeros(P, dtype=torch.int32, device=DEV)
    actkv.acquire_pages(bt[:2].contiguous(), refs)
    free = perm[2 * W:].contiguous()
    f = actkv.Forks([0, 0, 1, 1], [2, 3, 4, 5], [W - 3, W, 0, 7], [W, W, W, W]).to_device(DEV)
    ws = actkv.release_workspace(P, 4 * W)
    freed = torch.empty(4 * W, dtype=torch.int32, device=DEV)
    count = torch.empty(1, dtype=torch.int32, device=DEV)

    def body():
        actkv.fork_pages(f, kv, bt, free, refs)
        actkv.release_pages(bt[2:], refs, freed=freed, num_freed=count, ws=ws)
    refs0 = refs.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        body()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    want = torch.sort(free[:f.num_fresh]).values
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        body()
    for rep in range(4):
        freed.fill_(-7)
        count.fill_(-7)
        bt[2:] = -8
        kv[:, free[:f.num_fresh].long()] = 0
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(refs, refs0), rep
        assert int(count) == f.num_fresh and torch.equal(freed[:f.num_fresh], want), rep
        assert (freed[f.num_fresh:] == -1).all()
        assert torch.equal(kv[:, free[:3].long()], kv[:, bt[0, W - 3:].long()])
        assert torch.equal(kv[:, bt[4].long()], kv[:, bt[1].long()])
