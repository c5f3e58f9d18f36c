"""Refusals of the decode-step operators (actkv_attend, actkv_fork_pages, actkv_acquire_pages,
actkv_release_pages, actkv_token_logprobs), on the host: nothing here reaches a GPU."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2609_31395_amd import actkv

FAKE = 0x10000   # never dereferenced: every call below fails before any launch
INVALID, UNSUPPORTED, SMALL, PAGES = -1, -2, -3, -4


def problem(**over):
    kw = dict(seq_lens=[40, 17], q_lens=[1, 2], budgets=[0] * 4, num_q_heads=8, num_kv_heads=2, head_dim=64,
              num_pages=16, bt_stride=3)
    kw.update(over)
    return actkv.Problem(**kw)


def c_attend(p=None, mirrors=True, **over):
    p = problem() if p is None else p
    lib = actkv.load_library()
    c = p.cstruct()
    if mirrors:
        c.seq_lens_d = c.q_lens_d = FAKE
    a = dict(q=FAKE, q_stride=512, kv=FAKE, bt=FAKE, lens=None, k=None, v=None, stride=0, out=FAKE, lse=None,
             ws=FAKE, ws_bytes=1 << 30)
    a.update(over)
    return lib.actkv_attend(ctypes.byref(c), *a.values(), None)


def attend_bytes(p):
    n = ctypes.c_size_t()
    code = actkv.load_library().actkv_attend_workspace(ctypes.byref(p.cstruct()), ctypes.byref(n))
    return code, n.value


@pytest.mark.parametrize("over,code", [
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(kv=None), INVALID), (dict(bt=None), INVALID),
    (dict(ws=None), INVALID), (dict(q_stride=504), INVALID), (dict(q_stride=516), INVALID),
    (dict(q=FAKE + 8), INVALID), (dict(out=FAKE + 2), INVALID), (dict(kv=FAKE + 4), INVALID),
    (dict(ws=FAKE + 8), INVALID), (dict(k=FAKE), INVALID), (dict(v=FAKE), INVALID),
    (dict(k=FAKE, v=FAKE, stride=64), INVALID), (dict(k=FAKE, v=FAKE, stride=132), INVALID),
    (dict(k=FAKE + 8, v=FAKE, stride=128), INVALID), (dict(k=FAKE, v=FAKE, stride=1 << 27), UNSUPPORTED),
    (dict(ws_bytes=64), SMALL), (dict(mirrors=False), INVALID),
])
def test_attend_refuses(over, code):
    assert c_attend(**over) == code


@pytest.mark.parametrize("over,code", [
    (dict(q_lens=[1, 17], seq_lens=[40, 17]), UNSUPPORTED),                     # 68 rows
    (dict(num_q_heads=130), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(page_size=32), UNSUPPORTED),
    (dict(q_lens=[41, 1]), INVALID), (dict(bt_stride=2), INVALID),
])
def test_attend_refuses_problems(over, code):
    p = problem(**over)
    assert attend_bytes(p)[0] == code and c_attend(p) == code


def test_attend_refuses_requests_past_the_entry_numbers():
    for length, code in ((1 << 30, 0), ((1 << 30) + 1, UNSUPPORTED), ((1 << 31) - 1, UNSUPPORTED)):
        p = problem(seq_lens=[length], q_lens=[1], budgets=[0], num_kv_heads=1, bt_stride=1 << 27)
        assert attend_bytes(p)[0] == code
        assert c_attend(p, ws_bytes=64) == (code or SMALL)


def test_attend_workspace_is_the_limit():
    code, need = attend_bytes(problem())
    assert code == 0 and need > 0
    assert c_attend(ws_bytes=need - 1) == SMALL
    assert actkv.load_library().actkv_attend_workspace(None, None) == INVALID
    # no token, no kernel: a call without work returns before any launch
    assert c_attend(problem(q_lens=[0, 0])) == 0


def test_attend_binding_checks_its_tensors():
    p = problem()
    p.seq_lens_d, p.q_lens_d, p.budgets_d = (torch.from_numpy(x.copy()) for x in (p.seq_lens, p.q_lens, p.budgets))
    bf = torch.bfloat16
    ok = dict(q=torch.zeros(3, 8, 64, dtype=bf), kv_cache=torch.zeros(2, 16, 16, 2, 64, dtype=bf),
              block_table=torch.zeros(2, 3, dtype=torch.int32), kv_lens=torch.zeros(4, dtype=torch.int32),
              k_new=torch.zeros(3, 2, 64, dtype=bf), v_new=torch.zeros(3, 2, 64, dtype=bf),
              out=torch.zeros(3, 8, 64, dtype=bf), lse=torch.zeros(3, 8),
              ws=torch.zeros(attend_bytes(p)[1], dtype=torch.uint8))
    with pytest.raises(ValueError, match="on the GPU"):
        actkv.attend(p, **ok)
    fused = torch.zeros(3, 12, 64, dtype=bf)   # q, k and v as parts of one projection
    with pytest.raises(ValueError, match="on the GPU"):
        actkv.attend(p, **{**ok, "q": fused[:, :8], "k_new": fused[:, 8:10], "v_new": fused[:, 10:]})
    for key, bad in [("q", torch.zeros(3, 8, 64)), ("q", torch.zeros(2, 8, 64, dtype=bf)),
                     ("q", torch.zeros(3, 64, 8, dtype=bf).transpose(1, 2)), ("q", None),
                     ("q", torch.zeros(1, 8, 64, dtype=bf).expand(3, 8, 64)),
                     ("kv_cache", ok["kv_cache"][:, :15].contiguous()), ("kv_cache", ok["kv_cache"][:, ::2]),
                     ("kv_cache", None), ("block_table", ok["block_table"].long()), ("block_table", ok["block_table"][:1]),
                     ("kv_lens", torch.zeros(3, dtype=torch.int32)), ("kv_lens", torch.zeros(4)),
                     ("k_new", None), ("v_new", None), ("v_new", fused[:, 10:]),
                     ("k_new", torch.zeros(3, 2, 32, dtype=bf)), ("out", torch.zeros(3, 8, 64)),
                     ("out", torch.zeros(3, 8, 63, dtype=bf)), ("lse", torch.zeros(23)), ("lse", torch.zeros(3, 8).double()),
                     ("ws", ok["ws"][:-1])]:
        with pytest.raises((ValueError, TypeError)) as e:
            actkv.attend(p, **{**ok, key: bad})
        assert "on the GPU" not in str(e.value), key


def c_fork(forks, rows=6, stride=4, **over):
    host = np.ascontiguousarray(np.array(forks, dtype=np.int32).reshape(-1, 4))
    a = dict(h=host.ctypes.data, d=FAKE, n=len(host), rows=rows, stride=stride, heads=2, dim=64, page=16, pages=32,
             kv=FAKE, bt=FAKE, free=FAKE, num_free=100, refs=FAKE)
    a.update(over)
    return actkv.load_library().actkv_fork_pages(*a.values(), None)


@pytest.mark.parametrize("forks,over,code", [
    ([[0, 6, 1, 2]], {}, INVALID), ([[6, 0, 1, 2]], {}, INVALID), ([[-1, 0, 1, 2]], {}, INVALID),
    ([[0, -1, 1, 2]], {}, INVALID), ([[0, 1, 3, 2]], {}, INVALID), ([[0, 1, -1, 2]], {}, INVALID),
    ([[0, 1, 1, 5]], {}, INVALID), ([[0, 0, 1, 2]], {}, INVALID),
    ([[0, 1, 1, 2], [0, 1, 1, 2]], {}, INVALID),       # a child of two forks
    ([[0, 1, 1, 2], [1, 2, 1, 2]], {}, INVALID),       # a child that is a parent
    ([[1, 2, 1, 2], [0, 1, 1, 2]], {}, INVALID),
    ([[0, 1, 0, 4], [0, 2, 1, 4]], dict(num_free=6), PAGES),
    ([[0, 1, 0, 1]], dict(free=None), INVALID), ([[0, 1, 0, 1]], dict(kv=None), INVALID),
    ([[0, 1, 0, 1]], dict(kv=FAKE + 8), INVALID), ([[0, 1, 1, 1]], dict(bt=None), INVALID),
    ([[0, 1, 1, 1]], dict(d=None), INVALID), ([[0, 1, 1, 1]], dict(h=None), INVALID),
    ([[0, 1, 1, 1]], dict(dim=96), UNSUPPORTED), ([[0, 1, 1, 1]], dict(page=32), UNSUPPORTED),
    ([[0, 1, 1, 1]], dict(heads=65), UNSUPPORTED), ([[0, 1, 1, 1]], dict(heads=0), INVALID),
    ([[0, 1, 1, 1]], dict(pages=0), INVALID), ([[0, 1, 1, 1]], dict(n=65536), UNSUPPORTED),
    ([[0, 1, 1, 1]], dict(stride=1 << 24), UNSUPPORTED), ([[0, 1, 1, 1]], dict(n=-1), INVALID), ([[0, 1, 1, 1]], dict(rows=-1), INVALID),
])
def test_fork_refuses(forks, over, code):
    assert c_fork(forks, **over) == code


def test_no_fork_needs_nothing():
    assert c_fork([[0, 1, 1, 1]], n=0, h=None, d=None, kv=None, bt=None, free=None, refs=None) == 0


def test_counts_refuse():
    lib = actkv.load_library()
    assert lib.actkv_acquire_pages(None, 3, 8, FAKE, None) == INVALID
    assert lib.actkv_acquire_pages(FAKE, 3, 8, None, None) == INVALID
    assert lib.actkv_acquire_pages(FAKE, -1, 8, FAKE, None) == INVALID
    assert lib.actkv_acquire_pages(FAKE, 3, 0, FAKE, None) == INVALID
    assert lib.actkv_acquire_pages(None, 0, 8, None, None) == 0
    n = ctypes.c_size_t()
    assert lib.actkv_release_workspace(-1, 8, ctypes.byref(n)) == INVALID
    assert lib.actkv_release_workspace(1, 1 << 31, ctypes.byref(n)) == UNSUPPORTED
    assert lib.actkv_release_workspace(1 << 31, 100, ctypes.byref(n)) == UNSUPPORTED
    assert lib.actkv_release_workspace(5, 100, ctypes.byref(n)) == 0

    def release(pages=FAKE, n_=5, row=0, num_pages=100, refs=FAKE, freed=2 * FAKE, count=FAKE, ws=FAKE, size=n.value):
        return lib.actkv_release_pages(pages, n_, row, num_pages, refs, freed, count, ws, size, None)
    for over in (dict(pages=None), dict(refs=None), dict(freed=None), dict(count=None), dict(ws=None),
                 dict(ws=FAKE + 2), dict(n_=-1), dict(row=-1), dict(num_pages=0), dict(freed=FAKE)):
        assert release(**over) == INVALID, over
    assert release(size=n.value - 1) == SMALL


def test_page_bindings_check_their_tensors():
    i32 = torch.int32
    pages, refs = torch.zeros(5, dtype=i32), torch.zeros(9, dtype=i32)
    for call in (lambda p, r: actkv.acquire_pages(p, r), lambda p, r: actkv.release_pages(p, r)):
        with pytest.raises(ValueError, match="on the GPU"):
            call(pages, refs)
        for p, r in [(None, refs), (pages.long(), refs), (torch.zeros(5, 2, dtype=i32)[:, 0], refs), (pages, None),
                     (pages, refs.long())]:
            with pytest.raises((ValueError, TypeError)) as e:
                call(p, r)
            assert "on the GPU" not in str(e.value)
    for kw in (dict(freed=torch.zeros(4, dtype=i32)), dict(num_freed=torch.zeros(0, dtype=i32)),
               dict(ws=torch.zeros(1, dtype=torch.uint8)), dict(freed=torch.zeros(5))):
        with pytest.raises((ValueError, TypeError)) as e:
            actkv.release_pages(pages, refs, **kw)
        assert "on the GPU" not in str(e.value)
    f = actkv.Forks([0], [1], [1], [2])
    f.device = torch.from_numpy(f.host.copy())
    ok = dict(kv_cache=torch.zeros(2, 9, 16, 2, 64, dtype=torch.bfloat16), block_table=torch.zeros(2, 3, dtype=i32),
              free_pages=torch.zeros(1, dtype=i32), refs=refs)
    with pytest.raises(ValueError, match="on the GPU"):
        actkv.fork_pages(f, **ok)
    for key, bad in [("kv_cache", ok["kv_cache"].view(-1)), ("kv_cache", None), ("kv_cache", ok["kv_cache"].float()),
                     ("kv_cache", ok["kv_cache"][:, ::2]), ("block_table", ok["block_table"].view(-1)),
                     ("block_table", ok["block_table"].long()), ("block_table", ok["block_table"][:, :2]),
                     ("free_pages", None), ("free_pages", torch.zeros(0, dtype=i32)), ("refs", refs[:8])]:
        with pytest.raises((ValueError, TypeError)) as e:
            actkv.fork_pages(f, **{**ok, key: bad})
        assert "on the GPU" not in str(e.value), key
    f.device = None
    with pytest.raises(ValueError, match="forks is required"):
        actkv.fork_pages(f, **ok)
    with pytest.raises(ValueError):
        actkv.Forks([0, 1], [1], [1], [2])
    with pytest.raises(ValueError):
        f.shared[0] = 0   # the device mirror would not follow


def c_logprobs(**over):
    a = dict(x=FAKE, type=0, rows=3, vocab=1000, stride=1000, tokens=FAKE, k=4, lp=FAKE, ent=FAKE, tt=FAKE, tl=FAKE,
             ws=FAKE, size=1 << 20)
    a.update(over)
    return actkv.load_library().actkv_token_logprobs(*a.values(), None)


@pytest.mark.parametrize("over,code", [
    (dict(x=None), INVALID), (dict(x=FAKE + 2), INVALID), (dict(x=FAKE + 1, type=1), INVALID), (dict(type=3), INVALID),
    (dict(type=-1), INVALID), (dict(rows=-1), INVALID), (dict(vocab=0), INVALID), (dict(stride=999), INVALID),
    (dict(tokens=None), INVALID), (dict(k=-1), INVALID), (dict(k=65), UNSUPPORTED), (dict(tt=None), INVALID),
    (dict(tl=None), INVALID), (dict(vocab=262145, stride=262145), UNSUPPORTED), (dict(rows=(1 << 20) + 1), UNSUPPORTED),
    (dict(ws=None), INVALID), (dict(ws=FAKE + 4), INVALID), (dict(size=8), SMALL),
])
def test_logprobs_refuses(over, code):
    assert c_logprobs(**over) == code


def test_logprobs_of_no_row_needs_nothing():
    assert c_logprobs(rows=0, x=None, tokens=None, ws=None, size=0) == 0


def test_logprobs_binding_checks_its_tensors():
    x, t = torch.zeros(3, 50), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="on the GPU"):
        actkv.token_logprobs(x, t, top_k=2)
    for args, kw in [((x[0], t), {}), ((x.double(), t), {}), ((x[:, ::2], t), {}), ((x[:1].expand(3, 50), t), {}),
                     ((x, t.int()), {}), ((x, t[:2]), {}), ((x, None), dict(logprobs=torch.zeros(3))),
                     ((x, t), dict(entropy=torch.zeros(2))), ((x, t), dict(top_k=2, top_tokens=torch.zeros(5, dtype=torch.int64))),
                     ((x, t), dict(top_k=2, top_logprobs=torch.zeros(6).double())), ((x, t), dict(ws=torch.zeros(3, dtype=torch.uint8)))]:
        with pytest.raises((ValueError, TypeError)) as e:
            actkv.token_logprobs(*args, **kw)
        assert "on the GPU" not in str(e.value)
    with pytest.raises(actkv.ActKVError):
        actkv.token_logprobs(x, t, top_k=65)
