"""The operators of a decode step that work on the same paged K/V cache as the compression, and
what a step's logits say: their plain forms, and the calls that an engine makes of this library.

  attend    attention of a request's newest tokens over its cache, with a length per KV head (what
            a compaction with unequal budgets leaves), their own K and V rows written first where
            the call brings them; the outputs and the log-sum-exp that scoring takes
  logprobs  the log probabilities of given tokens, the entropy of each row and its top
            alternatives
  branch    requests forked into branches (full pages shared and counted, the others copied), and
            the branches' pages released again

The cache is bf16 [2][pages][16][kv heads][head dim]; values are N(0, 1), 1% of the keys leaning
towards the mean query of their head, pages scattered over a pool larger than what is in use, as in
the repository's other synthetic inputs.  Lengths and budgets belong to the case (its `lens`), the
values to the seed.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
DEVICE = "cuda"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _attend(name, reqs, len_lo, len_hi, q_heads, kv_heads, head_dim, tokens=1, budget="whole",
            append=False, fused_qkv=False, lens=1):
    c = dict(kind="attend", reqs=reqs, len_lo=len_lo, len_hi=len_hi, q_heads=q_heads,
             kv_heads=kv_heads, head_dim=head_dim, tokens=tokens, budget=budget, append=append,
             fused_qkv=fused_qkv, lens=lens)
    if name:
        c["name"] = name
    return c


def _logprobs(name, rows, vocab, dtype, top, padded=0, masked=0.0):
    c = dict(kind="logprobs", rows=rows, vocab=vocab, dtype=dtype, top=top, padded=padded,
             masked=masked)
    if name:
        c["name"] = name
    return c


def _branch(name, parents, children, len_lo, len_hi, kv_heads, head_dim, budget="whole",
            share=True, lens=1):
    c = dict(kind="branch", parents=parents, children=children, len_lo=len_lo, len_hi=len_hi,
             kv_heads=kv_heads, head_dim=head_dim, budget=budget, share=share, lens=lens)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a decode step of four short conversations, the new token's K and V in the same call:
        # latency
        _attend("attend_short", 4, 2048, 2048, 32, 8, 128, append=True),
        # one agent trace of a 25-iteration web task: few segments, long ones
        _attend("attend_one_trace", 1, 35000, 35000, 32, 4, 128),
        # a batch that went through a compression with unequal head budgets: a length per head
        _attend("attend_compacted", 32, 8000, 40000, 32, 4, 128, budget="dirichlet", append=True,
                fused_qkv=True, lens=1004),
        # a few drafted tokens at a time over ragged traces, 64-element heads
        _attend("attend_draft", 16, 3000, 20000, 64, 8, 64, tokens=5, lens=77),
        # a decode step over the headline batch: 32 requests of 35,000 tokens
        _attend("attend_batch", 32, 35000, 35000, 32, 4, 128),
        # the token that one conversation sampled: a 16-bit head with a small vocabulary
        _logprobs("logprobs_one", 1, 32000, "fp16", 1),
        # a decode step's logits over a 151,936-token vocabulary, part of it masked by a grammar,
        # with the alternatives that a client asks for
        _logprobs("logprobs_step", 32, 151936, "fp32", 20, masked=0.3),
        # a prompt scored token by token, the head's output padded
        _logprobs("logprobs_prompt", 4000, 151936, "bf16", 0, padded=64),
        # one conversation branched four ways, the branches dropped again: latency
        _branch("branch_one", 1, 4, 2005, 2005, 8, 128),
        # a batch of traces branched eight ways: counts and tables of half a million pages
        _branch("branch_batch", 32, 8, 30000, 35000, 4, 128, lens=1006),
        # branches that own all their pages, as an in-place compaction needs: a copy
        _branch("branch_copied", 4, 2, 30000, 35000, 4, 128, budget="dirichlet", share=False,
                lens=1007),
    ]


HEADS = [(8, 2, 64), (32, 4, 128), (32, 8, 128), (64, 8, 64), (16, 8, 128), (16, 2, 128),
         (28, 4, 128), (12, 12, 64)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, never more work than the largest listed one."""
    kind = rng.choice(["attend", "attend", "attend", "logprobs", "logprobs", "branch"])
    lens = rng.randrange(1, 1 << 20)
    if kind == "logprobs":
        top = rng.choice([0, 1, 5, 20, 64])
        vocab = _log(rng, 1000, 200000)
        rows = _log(rng, 1, min(4000, int((6e8 if top == 0 else 4e7) / vocab)))
        return _logprobs(None, rows, vocab, rng.choice(["fp32", "bf16", "fp16"]) if rows * vocab < 2e8
                         else "bf16", top, rng.choice([0, 64]), rng.choice([0.0, 0.0, 0.3]))
    budget = rng.choice(["whole", "dirichlet"])
    while True:
        hq, hkv, d = rng.choice(HEADS)
        hi = _log(rng, 64, 64000)
        lo = hi if rng.random() < 0.3 else max(16, int(hi * rng.uniform(0.2, 0.9)))
        if kind == "branch":
            share = rng.random() < 0.6
            parents, children = _log(rng, 1, 32), _log(rng, 1, 8)
            c = _branch(None, parents, children, lo, hi, hkv, d, budget, share, lens)
            if parents * hi * hkv * d <= 2e8 and parents * hi * children <= 7e6 and work(c)["bytes"] <= 1.1e9:
                return c
        else:
            reqs = _log(rng, 1, 128)
            tokens = 1 if rng.random() < 0.7 else rng.randrange(2, 64 // (hq // hkv) + 1)
            if reqs * hi * hkv * d * max(1.0, tokens * (hq // hkv) / 16) <= 5.5e8 and tokens <= lo:
                return _attend(None, reqs, lo, hi, hq, hkv, d, tokens, budget, rng.random() < 0.5,
                               rng.random() < 0.5, lens)


def _shape(case):
    """Lengths [requests, kv heads] and newest tokens [requests] of a case (the same for every
    seed): whole, or what a compaction leaves of a Dirichlet(0.5) split of a quarter of the cache
    over its heads, and the newest tokens behind it."""
    rng = np.random.default_rng(case["lens"])
    R, H = case.get("reqs", case.get("parents")), case["kv_heads"]
    L = rng.integers(case["len_lo"], case["len_hi"] + 1, size=R)
    n = np.full(R, case.get("tokens", 0))
    if case["budget"] == "whole":
        return np.repeat(L[:, None], H, axis=1).astype(np.int32), n.astype(np.int32)
    w = rng.dirichlet(np.full(H, 0.5), size=R)
    kept = np.minimum(np.floor(w * H * 0.25 * L[:, None]), L[:, None])
    return (kept + n[:, None]).astype(np.int32), n.astype(np.int32)


class State:
    pass


def _pool(s, case, lens, extra_rows, fresh):
    """The cache, the block table (rows of extra_rows more requests at its end, empty) and the
    free list; `fresh` pages at least are free."""
    R, H, D = lens.shape[0], case["kv_heads"], case["head_dim"]
    pages = -(-lens.max(axis=1) // PAGE)
    used, width = int(pages.sum()), max(1, int(pages.max()))
    total = used + max(used // 4, fresh) + 1
    s.kv = torch.randn(2, total, PAGE, H, D, device=DEVICE, dtype=torch.bfloat16, generator=s.gen)
    perm = torch.randperm(total, device=DEVICE, generator=s.gen).int()
    s.table = torch.full((R + extra_rows, width), -1, dtype=torch.int32, device=DEVICE)
    at = torch.from_numpy(np.arange(width) < pages[:, None]).to(DEVICE)
    s.table[:R][at] = perm[:used]
    s.free = perm[used:].contiguous()
    s.pages = pages


def _prepare_attend(s, case):
    lens, n = _shape(case)
    R, H, D = case["reqs"], case["kv_heads"], case["head_dim"]
    Hq, N = case["q_heads"], int(n.sum())
    _pool(s, case, lens, 0, 0)
    # queries and the newest tokens' K and V: arrays of their own, or parts of the rows of one
    # fused projection
    row = torch.randn(N, Hq + 2 * H, D, device=DEVICE, dtype=torch.bfloat16, generator=s.gen)
    s.q, s.k_new, s.v_new = row[:, :Hq], row[:, Hq:Hq + H], row[:, Hq + H:]
    if not case["fused_qkv"]:
        s.q, s.k_new, s.v_new = s.q.contiguous(), s.k_new.contiguous(), s.v_new.contiguous()
    if not case["append"]:
        s.k_new = s.v_new = None
    s.lens = torch.from_numpy(lens).to(DEVICE)
    s.n = torch.from_numpy(n).to(DEVICE)
    s.tokens = case["tokens"]
    # 1% of the keys lean towards the mean query of their head
    T = s.table.shape[1] * PAGE
    r, t = torch.nonzero((torch.rand(R, T, device=DEVICE, generator=s.gen) < 0.01)
                         & (torch.arange(T, device=DEVICE) < s.lens.amax(1, keepdim=True)),
                         as_tuple=True)
    mean = s.q.float().view(R, s.tokens, H, Hq // H, D).mean((1, 3))
    at = s.table[r, t // PAGE].long()
    s.kv[0, at, t % PAGE] += 3 * mean[r].bfloat16()
    if own:
        from paper_2609_31395_amd import actkv
        s.call = actkv.attend
        s.problem = actkv.Problem(
            seq_lens=lens.max(axis=1), q_lens=n, budgets=lens.reshape(-1), num_q_heads=Hq,
            num_kv_heads=H, head_dim=D, num_pages=s.kv.shape[1], bt_stride=s.table.shape[1],
        ).to_device(DEVICE)
        s.kv_lens = s.lens.reshape(-1) if case["budget"] != "whole" else None
        s.ws = actkv.attend_workspace(s.problem, DEVICE)
        s.out = torch.empty(N, Hq, D, dtype=torch.bfloat16, device=DEVICE)
        s.lse = torch.empty(N, Hq, dtype=torch.float32, device=DEVICE)


def _run_attend(s, case):
    if own:
        out, lse = s.call(s.problem, s.q, s.kv, s.table, kv_lens=s.kv_lens, k_new=s.k_new,
                          v_new=s.v_new, out=s.out, lse=s.lse, ws=s.ws)
    else:
        out, lse = _plain_attend(s)
    return dict(out=out, lse=lse, kv=s.kv) if case["append"] else dict(out=out, lse=lse)


def _plain_attend(s):
    """softmax(q K^T / sqrt(D)) V per request and head; token j of n sees the entries up to
    its own place, len - n + j."""
    R, n = s.table.shape[0], s.tokens
    (_, _, _, H, D), Hq = s.kv.shape, s.q.shape[1]
    G, dev = Hq // H, s.kv.device
    place = s.lens[:, None, :] - n + torch.arange(n, device=dev)[None, :, None]   # [R, n, H]
    if s.k_new is not None:
        page = s.table[torch.arange(R, device=dev)[:, None, None], place // PAGE].long()
        head = torch.arange(H, device=dev).expand_as(place)
        s.kv[0, page, place % PAGE, head] = s.k_new.reshape(R, n, H, D)
        s.kv[1, page, place % PAGE, head] = s.v_new.reshape(R, n, H, D)
    at = s.table.long().clamp(min=0)
    k = s.kv[0][at].reshape(R, -1, H, D).permute(0, 2, 3, 1).float()
    q = s.q.reshape(R, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(R, H, n * G, D).float()
    x = torch.matmul(q, k) * (1.0 / math.sqrt(D))
    del k
    last = place.permute(0, 2, 1).repeat_interleave(G, dim=2)[..., None]          # [R, H, n G, 1]
    x = x.masked_fill(torch.arange(x.shape[-1], device=dev) > last, -math.inf)
    m = x.amax(-1, keepdim=True)
    x = torch.exp(x - m.clamp(min=-1e30))
    v = s.kv[1][at].reshape(R, -1, H, D).permute(0, 2, 1, 3).float()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x, v) / total.clamp(min=1e-30)
    lse = (m + torch.log(total)).reshape(R, H, n, G).permute(0, 2, 1, 3).reshape(R * n, Hq)
    return (o.reshape(R, H, n, G, D).permute(0, 2, 1, 3, 4).reshape(R * n, Hq, D).bfloat16(), lse)


def _exact_attend(s, case):
    lens, _ = _shape(case)
    n, H, D = case["tokens"], case["kv_heads"], case["head_dim"]
    Hq = case["q_heads"]
    G, cache = Hq // H, s.kv.clone() if case["append"] else s.kv
    out = torch.zeros(case["reqs"] * n, Hq, D, dtype=torch.float64, device=DEVICE)
    lse = torch.full((case["reqs"] * n, Hq), -math.inf, dtype=torch.float64, device=DEVICE)
    for r in range(case["reqs"]):
        rows = cache[:, s.table[r, :int(s.pages[r])].long()].reshape(2, -1, H, D)
        for h in range(H):
            L = int(lens[r, h])
            k, v = rows[0, :L, h].double(), rows[1, :L, h].double()
            if case["append"]:
                k[L - n:], v[L - n:] = s.k_new[r * n:r * n + n, h].double(), s.v_new[r * n:r * n + n, h].double()
                for j in range(n):
                    t = L - n + j
                    page = int(s.table[r, t // PAGE])
                    cache[0, page, t % PAGE, h] = s.k_new[r * n + j, h]
                    cache[1, page, t % PAGE, h] = s.v_new[r * n + j, h]
            for j in range(n):
                see = L - n + j + 1
                if see < 1:
                    continue
                x = k[:see] @ s.q[r * n + j, h * G:h * G + G].double().T / math.sqrt(D)
                out[r * n + j, h * G:h * G + G] = torch.softmax(x, 0).T @ v[:see]
                lse[r * n + j, h * G:h * G + G] = torch.logsumexp(x, 0)
    return dict(out=out, lse=lse, kv=cache) if case["append"] else dict(out=out, lse=lse)


def _prepare_logprobs(s, case):
    rows, vocab = case["rows"], case["vocab"]
    width = vocab if not case["padded"] else -(-vocab // case["padded"]) * case["padded"] + case["padded"]
    x = torch.randn(rows, width, device=DEVICE, dtype=DTYPES[case["dtype"]], generator=s.gen)
    x *= 3
    if case["masked"]:
        x.masked_fill_(torch.rand(rows, width, device=DEVICE, generator=s.gen) < case["masked"], -math.inf)
    s.logits = x[:, :vocab]
    # what a sampler took: the best of a few candidates
    few = torch.randint(0, vocab, (rows, 64), device=DEVICE, generator=s.gen)
    s.given = few.gather(1, s.logits.gather(1, few).float().argmax(1, keepdim=True)).reshape(-1)
    s.top = case["top"]
    if own:
        from paper_2609_31395_amd import actkv
        s.call = actkv.token_logprobs


def _run_logprobs(s, case):
    r = s.call(s.logits, s.given, top_k=s.top) if own else _plain_logprobs(s)
    names = ("logprobs", "entropy") + (("top_tokens", "top_logprobs") if s.top else ())
    return {k: r[k] for k in names}


def _plain_logprobs(s):
    """log p = x - log sum exp x; entropy = -sum p log p; the largest, ties to the lower token."""
    x = s.logits.float()
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    r = dict(logprobs=(x.gather(1, s.given[:, None]) - lse)[:, 0],
             entropy=(torch.log(total) - (e * (x - m).clamp(min=-1e30)).sum(1, keepdim=True) / total)[:, 0])
    if s.top:
        # order keys: the value's bits in the order of the values, then the lower token first
        bits = (x + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 20) - torch.arange(x.shape[1], device=x.device)
        r["top_tokens"] = torch.topk(key, s.top, 1).indices
        r["top_logprobs"] = x.gather(1, r["top_tokens"]) - lse
    return r


def _exact_logprobs(s, case):
    rows, top = case["rows"], case["top"]
    got = dict(logprobs=[], entropy=[], top_tokens=[], top_logprobs=[])
    for a in range(0, rows, 250):
        p = torch.log_softmax(s.logits[a:a + 250].double(), 1)
        got["logprobs"].append(p.gather(1, s.given[a:a + 250, None])[:, 0])
        got["entropy"].append(-torch.where(p > -math.inf, p * torch.exp(p), 0.0).sum(1))
        if top:
            o = torch.sort(s.logits[a:a + 250].double(), dim=1, descending=True, stable=True).indices[:, :top]
            got["top_tokens"].append(o)
            got["top_logprobs"].append(p.gather(1, o))
    return {k: torch.cat(v) for k, v in got.items() if v}


def _branches(case):
    """Parent, child, shared pages and pages of every branch."""
    lens, _ = _shape(case)
    P, C = case["parents"], case["children"]
    whole, pages = lens.min(axis=1) // PAGE, -(-lens.max(axis=1) // PAGE)
    parent = np.repeat(np.arange(P), C)
    return np.stack([parent, P + np.arange(P * C), whole[parent] if case["share"] else 0 * parent,
                     pages[parent]], axis=1).astype(np.int32), lens


def _prepare_branch(s, case):
    forks, lens = _branches(case)
    s.fresh = int((forks[:, 3] - forks[:, 2]).sum())
    _pool(s, case, lens, len(forks), s.fresh)
    P = case["parents"]
    s.refs = torch.zeros(s.kv.shape[1], dtype=torch.int32, device=DEVICE)
    s.refs[s.table[:P][s.table[:P] >= 0].long()] = 1
    s.forks = torch.from_numpy(forks).to(DEVICE)
    s.children = s.table[P:]
    if own:
        from paper_2609_31395_amd import actkv
        s.lib = actkv
        s.plan = actkv.Forks(parents=forks[:, 0], children=forks[:, 1], shared=forks[:, 2],
                             pages=forks[:, 3]).to_device(DEVICE)
        s.ws = actkv.release_workspace(s.refs.numel(), s.children.numel(), DEVICE)


def _run_branch(s, case):
    if own:
        s.lib.fork_pages(s.plan, s.kv, s.table, s.free, s.refs)
        freed, count = s.lib.release_pages(s.children, s.refs, ws=s.ws)
    else:
        freed, count = _plain_branch(s)
    return dict(table=s.table, refs=s.refs, freed=freed, count=count, kv=s.kv)


def _plain_branch(s):
    parent, child, shared, pages = (v[:, None].long() for v in s.forks.unbind(1))
    # fork: the shared pages counted, the others copied into fresh ones
    col = torch.arange(s.table.shape[1], device=s.table.device)
    source = s.table[parent[:, 0]].long()
    kept, copied = col < shared, (col >= shared) & (col < pages)
    before = torch.cumsum(pages - shared, 0) - (pages - shared)
    place = (before + col - shared).clamp(0, s.free.numel() - 1)
    row = torch.where(kept, source, torch.where(copied, s.free[place].long(), -1))
    s.table[child[:, 0]] = row.int()
    s.refs.index_add_(0, source.clamp(min=0).reshape(-1), kept.reshape(-1).int())
    s.refs[s.free[:s.fresh].long()] = 1
    fork = torch.repeat_interleave(torch.arange(child.shape[0], device=col.device),
                                   (pages - shared)[:, 0], output_size=s.fresh)
    at = torch.arange(s.fresh, device=col.device) - before[fork, 0] + shared[fork, 0]
    s.kv[:, s.free[:s.fresh].long()] = s.kv[:, source[fork, at]]
    # release: one count off for every entry, the pages that nobody holds listed in their order
    entries = s.children.reshape(-1).long()
    off = torch.zeros_like(s.refs).index_add_(0, entries.clamp(min=0), (entries >= 0).int())
    gone = (s.refs > 0) & (s.refs <= off)
    s.refs.copy_((s.refs - off).clamp(min=0))
    place = torch.cumsum(gone, 0) - 1
    freed = torch.full((entries.numel() + 1,), -1, dtype=torch.int32, device=col.device)
    freed[torch.where(gone, place, entries.numel())] = torch.where(
        gone, torch.arange(gone.numel(), device=col.device), -1).int()
    return freed[:-1], gone.sum().reshape(1).int()


def _exact_branch(s, case):
    """The copies in their places (whole numbers are compared as they are)."""
    forks, _ = _branches(case)
    free, table, at = s.free.cpu().numpy(), s.table.cpu().numpy(), 0
    cache = s.kv.clone()
    for parent, _, shared, pages in forks:
        m = int(pages - shared)
        cache[:, torch.from_numpy(free[at:at + m]).long().to(DEVICE)] = s.kv[
            :, torch.from_numpy(table[parent, shared:pages]).long().to(DEVICE)]
        at += m
    return dict(table=None, refs=None, freed=None, count=None, kv=cache)


def prepare(case, seed):
    s = State()
    s.gen = torch.Generator(device=DEVICE).manual_seed(int(seed) * 1000003 + 17)
    dict(attend=_prepare_attend, logprobs=_prepare_logprobs, branch=_prepare_branch)[case["kind"]](s, case)
    s.case = case
    return s


def run(state):
    return dict(attend=_run_attend, logprobs=_run_logprobs, branch=_run_branch)[state.case["kind"]](
        state, state.case)


def exact(case, seed):
    return dict(attend=_exact_attend, logprobs=_exact_logprobs, branch=_exact_branch)[case["kind"]](
        prepare(case, seed), case)


def work(case):
    if case["kind"] == "logprobs":
        n = case["rows"] * case["vocab"]
        size = 4 if case["dtype"] == "fp32" else 2
        return dict(bytes=n * size + case["rows"] * (16 + 12 * case["top"]), flops=4 * n)
    H, D = case["kv_heads"], case["head_dim"]
    if case["kind"] == "branch":
        forks, lens = _branches(case)
        pages = int(forks[:, 3].sum())
        fresh = int((forks[:, 3] - forks[:, 2]).sum())
        # K and V of the copied pages read and written; the parents' rows read, the branches' rows
        # written and read, a count read and written for each entry by the fork and by the release,
        # the freed list
        rows = int((-(-lens.max(axis=1) // PAGE)).sum())
        return dict(bytes=fresh * 2 * 2 * PAGE * H * D * 2 + 4 * rows + 8 * pages + 16 * pages + 8 * fresh,
                    flops=0)
    lens, n = _shape(case)
    entries, new = int(lens.sum(dtype=np.int64)), int(n.sum())
    Hq = case["q_heads"]
    size = entries * 2 * D * 2 + new * Hq * (4 * D + 4) + int((-(-lens.max(axis=1) // PAGE)).sum()) * 4
    if case["append"]:
        size += new * H * 2 * D * 2   # written; read they are as entries
    return dict(bytes=size, flops=int((lens.sum(axis=1) * n).sum()) * (Hq // H) * D * 4)
