"""Cases of the operators around the sparse decode: attention of whole prompts, dense
attention of a new token over a paged cache, and the upkeep of that cache's pages.

A case is a dict of plain values:
  op     "prompt"   causal attention of packed prompts; kv: where the keys are --
                    "packed" (K and V are parts of one fused projection's rows), "cache"
                    (the contiguous caches [B, Hkv, L_max, d] of the decode calls) or
                    "paged" (a prompt's next part over the pages of what came before)
         "decode"   one new token of every sequence over paged caches, with `append`
                    preceded by writing the token's K and V rows into their pages
         "branch"   the branches of some sequences are dropped, forked anew from their
                    parents, the parents' half-filled last pages copied in every layer,
                    and room for the branches' next tokens taken
         "compact"  live pages of a pool moved together at its front
  n      sequences (branch: branches)
  Hq, Hkv         query and KV heads (head dimension 128)
  q_lo, q_hi      new tokens of a sequence, from .. to       (prompt)
  kv_lo, kv_hi    tokens of a sequence before those           (prompt)
                  cached tokens of a sequence                 (decode, branch, compact)
  P      tokens of a page
  dtype  "float16" or "bfloat16"
  layers pools that the page copies of a branch go through
  spread which of the lengths in a range the sequences have (a seed of their own: the
         lengths belong to the case, the values to the inputs)
"""
import math
import random

import torch

own = False

D = 128
N_OUTLIER, OUTLIER_SCALE = 8, 8.0      # channels of K that are large in every token, as in the workloads


def _prompt(n, Hq, Hkv, q_lo, q_hi, kv="packed", kv_lo=0, kv_hi=0, P=16, dtype="float16", spread=0):
    return {"op": "prompt", "n": n, "Hq": Hq, "Hkv": Hkv, "q_lo": q_lo, "q_hi": q_hi, "kv": kv,
            "kv_lo": kv_lo, "kv_hi": kv_hi, "P": P, "dtype": dtype, "spread": spread}


def _decode(n, Hq, Hkv, kv_lo, kv_hi, P=16, dtype="float16", append=False, spread=0):
    return {"op": "decode", "n": n, "Hq": Hq, "Hkv": Hkv, "kv_lo": kv_lo, "kv_hi": kv_hi, "P": P,
            "dtype": dtype, "append": append, "spread": spread}


def _branch(n, Hkv, kv_lo, kv_hi, P=16, layers=1, n_new=1, dtype="float16", spread=0):
    return {"op": "branch", "n": n, "Hkv": Hkv, "kv_lo": kv_lo, "kv_hi": kv_hi, "P": P, "layers": layers,
            "n_new": n_new, "dtype": dtype, "spread": spread}


def _compact(n, Hkv, kv_lo, kv_hi, P=16, dtype="float16", spread=0):
    return {"op": "compact", "n": n, "Hkv": Hkv, "kv_lo": kv_lo, "kv_hi": kv_hi, "P": P, "dtype": dtype, "spread": spread}


def listed():
    named = {
        # a question of some words, alone: latency
        "prompt_97": _prompt(1, 32, 32, 97, 97),
        # prompts that came in together, of a word up to a few pages, packed without padding
        "prompts_packed": _prompt(11, 32, 8, 1, 2300, dtype="bfloat16", spread=3),
        # the long prompt that the contiguous caches of a sparse decode start from, the 7B shape
        "prompt_8k_cache": _prompt(1, 32, 32, 8192, 8192, kv="cache"),
        # two long documents, grouped queries: the largest amount of arithmetic
        "prompts_2x8k": _prompt(2, 32, 8, 8100, 8192, dtype="bfloat16", spread=1),
        # the next 512 tokens of two prompts that are taken in by parts, over their pages
        "part_512_over_20k": _prompt(2, 64, 8, 512, 512, kv="paged", kv_lo=15000, kv_hi=20011, spread=2),
        # a short conversation's next token
        "token_900": _decode(1, 32, 32, 907, 907),
        # a server's batch: conversations of a few tokens up to long ones, the new rows written first
        "tokens_ragged": _decode(48, 32, 8, 3, 20000, dtype="bfloat16", append=True, spread=5),
        # the 70B shape at batch 16, pages of 64 tokens: the largest amount of memory
        "tokens_16x32k": _decode(16, 64, 8, 32000, 32768, P=64, spread=4),
        # one conversation of 256K tokens
        "token_250k": _decode(1, 28, 4, 250007, 250007, P=32),
        # one conversation is branched
        "branch_1": _branch(1, 8, 1001, 1001),
        # beams of a batch, 16 layers' pools
        "branch_64": _branch(64, 8, 100, 6000, layers=16, n_new=5, spread=6),
        # a pool in which half of the sequences have ended is closed up
        "compact_2gib": _compact(40, 8, 50, 14000, dtype="bfloat16", spread=7),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_SCORES = 1 << 32       # of a padded batch of prompts, all heads
MOST_KV = 1 << 31           # bytes of K and V that a decode reads


def draw(rng):
    op = rng.choices(("prompt", "decode", "branch", "compact"), (5, 5, 1, 1))[0]
    while True:
        Hq, Hkv = rng.choice(((32, 32), (8, 8), (40, 40), (32, 16), (32, 8), (64, 8), (28, 4), (32, 2)))
        P = rng.choice((16, 16, 32, 64, 128))
        dtype = rng.choice(("float16", "bfloat16"))
        spread = rng.randrange(1 << 20)
        if op == "prompt":
            n, hi = _log(rng, 1, 32), _log(rng, 16, 8192)
            lo = hi if rng.random() < 0.3 else max(1, hi // rng.choice((2, 8, 64)))
            kv = rng.choice(("packed", "packed", "cache", "paged"))
            before = _log(rng, 1, 32768) if kv != "packed" and rng.random() < 0.7 else 0
            c = _prompt(n, Hq, Hkv, lo, hi, kv, before // 2, before, P, dtype, spread)
            fits = n * Hq * hi * (hi + before) <= MOST_SCORES and work(c)["flops"] <= work(listed()[3])["flops"]
        elif op == "decode":
            n, hi = _log(rng, 1, 128), _log(rng, 16, 262144)
            lo = max(1, hi // rng.choice((1, 2, 8, 64, 1024)))
            c = _decode(n, Hq, Hkv, lo, hi, P, dtype, rng.random() < 0.4, spread)
            fits = n * hi * Hkv * D * 4 <= MOST_KV
        elif op == "branch":
            n, hi = _log(rng, 1, 128), _log(rng, 16, 8192)
            c = _branch(n, rng.choice((2, 4, 8, 32)), max(1, hi // rng.choice((1, 4, 64))), hi, P, _log(rng, 1, 16),
                        rng.choice((1, 1, 5, 40)), dtype, spread)
            fits = work(c)["bytes"] <= work(listed()[10])["bytes"] and _pool_pages(c) * P * c["Hkv"] * D * 4 * c["layers"] <= 1 << 34
        else:
            n, hi = _log(rng, 2, 128), _log(rng, 64, 16384)
            c = _compact(n, rng.choice((2, 4, 8, 32)), max(1, hi // rng.choice((2, 16, 64))), hi, P, dtype, spread)
            fits = _pool_pages(c) * P * c["Hkv"] * D * 4 <= MOST_KV
        if fits:
            return c


# ------------------------------------------------------------------ lengths and pages of a case
def _between(case, lo, hi, salt):
    """n lengths from lo to hi, over their logarithm; the longest is hi."""
    rng = random.Random(case["spread"] * 16 + salt)
    got = [min(hi, max(lo, _log(rng, max(lo, 1), max(hi, 1)))) if hi else 0 for _ in range(case["n"])]
    got[rng.randrange(len(got))] = hi
    return got


def _lengths(case):
    """(new tokens, tokens with those) of the sequences."""
    if case["op"] == "prompt":
        new = _between(case, case["q_lo"], case["q_hi"], 1)
        return new, [a + b for a, b in zip(new, _between(case, case["kv_lo"], case["kv_hi"], 2))]
    return [1] * case["n"], _between(case, case["kv_lo"], case["kv_hi"], 1)


def _pages_of(tokens, P):
    return (tokens + P - 1) // P


def _pool_pages(case):
    """Pages of the case's pool: what the sequences hold and an eighth more; branches: room for
    them too; compact: as much again, from sequences that have ended."""
    total = sum(_pages_of(x, case["P"]) for x in _lengths(case)[1])
    if case["op"] == "branch":
        total += case["n"] * (2 + _pages_of(case["n_new"], case["P"])) + sum(_pages_of(x, case["P"]) for x in _lengths(case)[1]) // 2
    if case["op"] == "compact":
        total = total * 9 // 5
    return total + total // 8 + 1


# ------------------------------------------------------------------ inputs
class _State:
    pass


def _rand(g, shape, dtype, scale=None):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    if scale is not None:
        x.mul_(scale)
    return x.to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _fill_pool(g, n_pages, Hkv, P, dtype, scale):
    """A pool [n_pages + 1, Hkv, P, d] (the last page is nobody's: the plain form's writes to nowhere go there)."""
    pool = torch.empty((n_pages + 1, Hkv, P, D), dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // (Hkv * P * D))
    for p in range(0, n_pages + 1, step):
        part = pool[p:p + step]
        part.copy_(_rand(g, part.shape, dtype, scale))
    return pool


def _paged(s, c, g, scale, layers=1):
    """Pools and a page table over a shuffled pool: what a server has after some hours."""
    P, n = c["P"], c["n"]
    s.n_pages = _pool_pages(c)
    s.pools = []
    for _ in range(layers):
        s.pools.append((_fill_pool(g, s.n_pages, c["Hkv"], P, s.dtype, scale), _fill_pool(g, s.n_pages, c["Hkv"], P, s.dtype, None)))
    order = torch.randperm(s.n_pages, generator=g, device="cuda").to(torch.int32)
    held = [_pages_of(x, P) for x in s.total]
    rows = 2 * n if c["op"] == "branch" else n
    s.max_pages = max(held) + _pages_of(c.get("n_new", 1), P) + 1
    s.table = torch.full((rows, s.max_pages), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, k in enumerate(held):
        s.table[i, :k] = order[at:at + k]
        at += k
    s.refs = torch.zeros(s.n_pages, dtype=torch.int32, device="cuda")
    s.refs[order[:at].long()] = 1
    s.lens = torch.zeros(rows, dtype=torch.int32, device="cuda")
    s.lens[:n] = _ints(s.total)
    return order, at


def prepare(case, seed):
    c, s = case, _State()
    s.case, s.ws = c, None
    s.dtype = getattr(torch, c["dtype"])
    g = torch.Generator(device="cuda")
    g.manual_seed(seed & 0x7FFFFFFFFFFF)
    Hkv, n = c["Hkv"], c["n"]
    s.new, s.total = _lengths(c)
    large = torch.rand((Hkv, D), generator=g, device="cuda").argsort(dim=1)[:, :N_OUTLIER]
    scale = torch.ones((Hkv, D), device="cuda").scatter_(1, large, OUTLIER_SCALE)
    paged_scale = scale[None, :, None, :]
    if c["op"] == "prompt":
        T = sum(s.new)
        s.q_start = _ints([sum(s.new[:i]) for i in range(n + 1)])
        s.kv_len = _ints(s.total)
        s.out = torch.zeros((T, c["Hq"], D), dtype=s.dtype, device="cuda")
        if c["kv"] == "packed":
            heads = c["Hq"] + 2 * Hkv
            fused = _rand(g, (T, heads, D), s.dtype)
            s.q, s.K, s.V = fused[:, :c["Hq"]], fused[:, c["Hq"]:c["Hq"] + Hkv], fused[:, c["Hq"] + Hkv:]
            s.K.copy_((s.K.float() * scale).to(s.dtype))
            s.kv_start = s.q_start[:n].clone()
        else:
            s.q = _rand(g, (T, c["Hq"], D), s.dtype)
            if c["kv"] == "cache":
                s.L_max = (max(s.total) + 63) // 64 * 64
                s.K = _rand(g, (n, Hkv, s.L_max, D), s.dtype, scale[None, :, None, :])
                s.V = _rand(g, (n, Hkv, s.L_max, D), s.dtype)
                s.kv_start = _ints([i * Hkv * s.L_max for i in range(n)])
            else:
                _paged(s, c, g, paged_scale)
    elif c["op"] == "decode":
        _paged(s, c, g, paged_scale)
        s.q = _rand(g, (n, c["Hq"], D), s.dtype)
        s.out = torch.zeros((n, c["Hq"], D), dtype=torch.float32, device="cuda")
        if c["append"]:
            s.k_new = _rand(g, (n, Hkv, D), s.dtype, scale)
            s.v_new = _rand(g, (n, Hkv, D), s.dtype)
            s.new_start = _ints(list(range(n + 1)))
            s.start = _ints([x - 1 for x in s.total])
    elif c["op"] == "branch":
        order, at = _paged(s, c, g, paged_scale, c["layers"])
        # rows n .. 2n are the branches; each still holds an older one: half of its parent's pages, of its own
        s.src, s.dst = _ints(list(range(n))), _ints(list(range(n, 2 * n)))
        for i, x in enumerate(s.total):
            k = _pages_of(x // 2, c["P"])
            s.table[n + i, :k] = order[at:at + k]
            s.refs[order[at:at + k].long()] = 1
            at += k
        s.lens[n:] = _ints([x // 2 for x in s.total])
        s.n_new = _ints([c["n_new"]] * n)
        s.copies = torch.zeros((n, 4), dtype=torch.int32, device="cuda")
        s.n_copies = torch.zeros(1, dtype=torch.int32, device="cuda")
        s.start = torch.zeros(n, dtype=torch.int32, device="cuda")
        s.status = torch.zeros(3, dtype=torch.int32, device="cuda")
    else:
        _paged(s, c, g, paged_scale)
        s.copies = torch.zeros((s.n_pages // 2 + 1, 4), dtype=torch.int32, device="cuda")
        s.n_copies = torch.zeros(1, dtype=torch.int32, device="cuda")
        s.status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    return s


def run(state):
    s, op = state, state.case["op"]
    if op == "prompt":
        return _own_prompt(s) if own else _plain_prompt(s)
    if op == "decode":
        return _own_decode(s) if own else _plain_decode(s)
    if op == "branch":
        return _own_branch(s) if own else _plain_branch(s)
    # the bookkeeping from before the pass stays as it was: a pass closes up a copy of it
    refs, table = s.refs.clone(), s.table.clone()
    return _own_compact(s, refs, table) if own else _plain_compact(s, refs, table)


# ------------------------------------------------------------------ the framework's calls
def _pages_arg(ds, s):
    c = s.case
    return ds.pages(s.n_pages, c["P"], c["Hkv"], D, s.table.shape[0], s.max_pages,
                    ds.DS_BF16 if s.dtype == torch.bfloat16 else ds.DS_F16)


def _own_prompt(s):
    import paper_2408_07092_amd as ds
    c = s.case
    if s.ws is None:
        more = {}
        if c["kv"] == "packed":
            row = s.q.stride(0)
            more = {"q_stride": row, "kv_stride": row, "kv_head_stride": D, "kv_elems": (s.q.shape[0] - 1) * row + c["Hkv"] * D}
        elif c["kv"] == "cache":
            more = {"kv_stride": D, "kv_head_stride": s.L_max * D, "kv_elems": s.K.numel()}
        s.prm = ds.prompt(c["n"], c["Hq"], c["Hkv"], D, s.q.shape[0], max(s.total),
                          ds.DS_BF16 if s.dtype == torch.bfloat16 else ds.DS_F16, **more)
        s.ws = ds.ds_prompt_workspace_alloc(s.prm)
        s.pages = _pages_arg(ds, s) if c["kv"] == "paged" else None
    if c["kv"] == "paged":
        ds.ds_prompt_attention_paged(s.q, s.pools[0][0], s.pools[0][1], s.out, s.q_start, None, s.lens, s.table, s.ws, s.prm, s.pages)
    else:
        ds.ds_prompt_attention(s.q, s.K, s.V, s.out, s.q_start, s.kv_start, s.kv_len, s.ws, s.prm)
    return {"out": s.out}


def _own_decode(s):
    import paper_2408_07092_amd as ds
    c = s.case
    if s.ws is None:
        s.pages = _pages_arg(ds, s)
        s.ws = ds.ds_paged_workspace_alloc(s.pages, c["n"], c["Hq"], max(s.total))
    K, V = s.pools[0]
    res = {}
    if c["append"]:
        ds.ds_append_paged(s.k_new, s.v_new, K, V, s.new_start, None, s.start, s.table, s.pages, c["n"])
        res["pools"] = [K, V]
    ds.ds_paged_decode(s.q, K, V, s.out, None, s.lens, s.table, s.ws, s.pages, c["n"], c["Hq"], max(s.total))
    res["out"] = s.out
    return res


def _own_branch(s):
    import paper_2408_07092_amd as ds
    c = s.case
    if s.ws is None:
        s.pages = _pages_arg(ds, s)
        s.ws = True
    ds.ds_pages_free(s.refs, s.table, s.lens, s.dst, s.status[0:1], s.pages, c["n"])
    ds.ds_pages_fork(s.refs, s.table, s.lens, s.src, s.dst, s.copies, s.n_copies, s.status[1:2], s.pages, c["n"])
    for K, V in s.pools:
        ds.ds_pages_copy(K, V, s.copies, s.n_copies, s.pages, c["n"])
    ds.ds_pages_extend(s.refs, s.table, s.lens, s.dst, s.n_new, s.start, s.status[2:3], s.pages, c["n"])
    return _branch_result(s)


def _own_compact(s, refs, table):
    import paper_2408_07092_amd as ds
    if s.ws is None:
        s.pages = _pages_arg(ds, s)
        s.ws = ds.ds_pages_workspace_alloc(s.pages)
    K, V = s.pools[0]
    ds.ds_pages_compact(refs, table, s.lens, s.copies, s.n_copies, s.status, s.ws, s.pages)
    ds.ds_pages_copy(K, V, s.copies, s.n_copies, s.pages, s.copies.shape[0])
    return _compact_result(s, refs, table)


# ------------------------------------------------------------------ the plain forms
def _branch_result(s):
    return {"refs": s.refs, "table": s.table, "lens": s.lens, "copies": s.copies, "n_copies": s.n_copies, "start": s.start,
            "status": s.status, "pools": [p[:s.n_pages] for kv in s.pools for p in kv]}


def _compact_result(s, refs, table):
    return {"refs": refs, "table": table, "copies": s.copies, "n_copies": s.n_copies, "status": s.status,
            "pools": [p[:s.n_pages] for p in s.pools[0]]}


def _padded_keys(s, top):
    """K and V of every sequence, [n, Hkv, top, d] in 32 bits, from wherever they are."""
    c = s.case
    n, Hkv, P = c["n"], c["Hkv"], c["P"]
    at = torch.arange(top, device="cuda")
    if c["op"] == "prompt" and c["kv"] == "packed":
        rows = (s.kv_start.long()[:, None] + at).clamp(max=s.K.shape[0] - 1)
        return [x[rows].permute(0, 2, 1, 3).float() for x in (s.K, s.V)]
    if c["op"] == "prompt" and c["kv"] == "cache":
        return [x[:, :, :top].float() for x in (s.K, s.V)]
    pages = s.table[:n, :_pages_of(top, P)].clamp(min=0).long()
    return [x[pages].permute(0, 2, 1, 3, 4).reshape(n, Hkv, -1, D)[:, :, :top].float() for x in s.pools[0]]


def _plain_attend(q, K, V, seen):
    """softmax(q K^T / sqrt(d)) V over the keys seen: q [n, Hkv, m, d], K and V [n, Hkv, t, d], seen [n, m]
    keys from the front; rows that see none are zero."""
    S = torch.matmul(q, K.transpose(2, 3)).mul_(1.0 / math.sqrt(D))
    hidden = torch.arange(K.shape[2], device="cuda") >= seen[:, :, None]
    S.masked_fill_(hidden[:, None], -math.inf)
    top = S.amax(dim=3, keepdim=True).clamp(min=-1e30)
    S.sub_(top).exp_()
    total = S.sum(dim=3, keepdim=True)
    return torch.matmul(S, V).div_(total.clamp(min=1e-30))


def _plain_prompt(s):
    c = s.case
    n, Hq, Hkv = c["n"], c["Hq"], c["Hkv"]
    G, m, top = Hq // Hkv, max(s.new), max(s.total)
    K, V = _padded_keys(s, top)
    q_start, new = s.q_start.long(), s.q_start.diff().long()
    at = torch.arange(m, device="cuda")
    rows = (q_start[:n, None] + at).clamp(max=s.q.shape[0] - 1)
    q = s.q[rows].float().reshape(n, m, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(n, Hkv, G * m, D)
    seen = (at + 1 + (s.kv_len.long() - new)[:, None]).clamp(min=0)
    O = _plain_attend(q, K, V, seen.repeat(1, G)).reshape(n, Hkv, G, m, D).permute(0, 3, 1, 2, 4)
    row = torch.arange(s.q.shape[0], device="cuda")
    seq = torch.searchsorted(q_start[1:].contiguous(), row, right=True)
    s.out.copy_(O[seq, row - q_start[seq]].reshape(-1, Hq, D))
    return {"out": s.out}


def _plain_decode(s):
    c = s.case
    n, Hq, Hkv, P = c["n"], c["Hq"], c["Hkv"], c["P"]
    res = {}
    if c["append"]:
        page = s.table[torch.arange(n, device="cuda"), s.start.long() // P].long()
        for pool, new in zip(s.pools[0], (s.k_new, s.v_new)):
            pool[page, :, s.start.long() % P] = new
        res["pools"] = list(s.pools[0])
    K, V = _padded_keys(s, max(s.total))
    q = s.q.float().reshape(n, Hkv, Hq // Hkv, D)
    s.out.copy_(_plain_attend(q, K, V, s.lens[:n].long()[:, None].expand(n, Hq // Hkv)).reshape(n, Hq, D))
    res["out"] = s.out
    return res


def _lowest_free(refs):
    return torch.sort((refs > 0).to(torch.int8), stable=True).indices


def _plain_copy(s, pools, used):
    """Rows of the listed pages, in every pool; entries past the count go to the page that is nobody's."""
    listed_ = torch.arange(s.copies.shape[0], device="cuda") < s.n_copies
    src = torch.where(listed_, s.copies[:, 0], s.n_pages).long()
    dst = torch.where(listed_, s.copies[:, 1], s.n_pages).long()
    kept = torch.arange(s.case["P"], device="cuda") >= used[:, None]
    for K in pools:
        K[dst] = torch.where(kept[:, None, :, None], K[dst], K[src])


def _plain_branch(s):
    c = s.case
    P, n = c["P"], c["n"]
    src, dst = s.src.long(), s.dst.long()
    slot = torch.arange(s.max_pages, device="cuda")
    # drop the old branches
    pages = s.table[dst].long()
    held = slot < _pages_of(s.lens[dst], P)[:, None]
    s.refs.index_add_(0, pages.clamp(min=0).flatten(), -held.to(torch.int32).flatten())
    s.table[dst] = torch.where(held, -1, s.table[dst])
    # fork: full pages shared, a half-filled last one to the lowest free page
    free = torch.cat((_lowest_free(s.refs), torch.zeros(1, dtype=torch.long, device="cuda")))
    length = s.lens[src]
    full, rest = length // P, length % P
    half = (rest > 0).to(torch.int32)
    rank = half.cumsum(0) - half
    fresh = free[rank]
    pages = s.table[src]
    shared = slot < full[:, None]
    s.refs.index_add_(0, pages.clamp(min=0).long().flatten(), shared.to(torch.int32).flatten())
    s.refs.index_add_(0, fresh, half)
    last = pages.gather(1, full.long()[:, None])[:, 0]
    entry = torch.stack((last, fresh.to(torch.int32), rest, torch.zeros_like(rest)), 1)
    copies = torch.cat((s.copies, s.copies[:1]))
    copies[torch.where(half > 0, rank, n).long()] = entry
    s.copies.copy_(copies[:n])
    s.n_copies.copy_(half.sum(dtype=torch.int32)[None])
    now = torch.where(shared, pages, s.table[dst])
    s.table[dst] = torch.where((slot == full[:, None]) & (half[:, None] > 0), fresh[:, None].to(torch.int32), now)
    s.lens[dst] = length
    _plain_copy(s, [p for kv in s.pools for p in kv], s.copies[:, 2])
    # room for the next tokens: the lowest free pages, ascending, branch after branch
    free = _lowest_free(s.refs)
    had, want = _pages_of(length, P), _pages_of(length + s.n_new, P)
    need = want - had
    rank = (need.cumsum(0) - need)[:, None] + slot - had[:, None]
    taken = (slot >= had[:, None]) & (slot < want[:, None])
    given = free[rank.clamp(0, s.n_pages - 1)]
    s.refs.index_add_(0, given.flatten(), taken.to(torch.int32).flatten())
    s.table[dst] = torch.where(taken, given.to(torch.int32), s.table[dst])
    s.start.copy_(length)
    s.lens[dst] = length + s.n_new
    s.status.zero_()
    return _branch_result(s)


def _plain_compact(s, refs, table):
    live = refs > 0
    n_live = live.sum()
    page = torch.arange(s.n_pages, device="cuda")
    mover = live & (page >= n_live)
    rank = mover.to(torch.int32).cumsum(0) - 1
    holes = _lowest_free(refs)
    to = torch.where(mover, holes[rank.clamp(min=0).long()], page)
    most = s.copies.shape[0]
    copies = torch.cat((s.copies, s.copies[:1]))
    entry = torch.stack((page, to, torch.full_like(page, s.case["P"]), torch.zeros_like(page)), 1).to(torch.int32)
    copies[torch.where(mover, rank, most).long()] = entry
    s.copies.copy_(copies[:most])
    s.n_copies.copy_(mover.sum(dtype=torch.int32)[None])
    held = torch.arange(s.max_pages, device="cuda") < _pages_of(s.lens, s.case["P"])[:, None]
    table.copy_(torch.where(held, to[table.clamp(min=0).long()].to(torch.int32), table))
    moved = torch.zeros_like(refs).index_add_(0, to, torch.where(live, refs, 0))
    refs.copy_(moved)
    _plain_copy(s, s.pools[0], s.copies[:, 2])
    s.status.zero_()
    return _compact_result(s, refs, table)


# ------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    c = case
    if c["op"] in ("branch", "compact"):
        return None         # whole numbers and copies
    s = prepare(case, seed)
    P, G = c["P"], c["Hq"] // c["Hkv"]
    if c["op"] == "decode" and c["append"]:
        for i, t in enumerate(s.start.tolist()):
            p = int(s.table[i, t // P])
            s.pools[0][0][p, :, t % P] = s.k_new[i]
            s.pools[0][1][p, :, t % P] = s.v_new[i]
    out = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda")
    row = 0
    for i, (nq, nk) in enumerate(zip(s.new, s.total)):
        for h in range(c["Hkv"]):
            if c["op"] == "prompt" and c["kv"] == "packed":
                k, v = (x[row:row + nk, h].double() for x in (s.K, s.V))
            elif c["op"] == "prompt" and c["kv"] == "cache":
                k, v = (x[i, h, :nk].double() for x in (s.K, s.V))
            else:
                used = s.table[i, :_pages_of(nk, P)].long()
                k, v = (x[used, h].reshape(-1, D)[:nk].double() for x in s.pools[0])
            first = torch.arange(nq, device="cuda") + (nk - nq)
            for j in range(h * G, (h + 1) * G):
                logit = s.q[row:row + nq, j].double() @ k.T / math.sqrt(D)
                if nq > 1:
                    logit = logit.masked_fill(torch.arange(nk, device="cuda") > first[:, None], -math.inf)
                out[row:row + nq, j] = torch.softmax(logit, dim=1) @ v
        row += nq
    res = {"out": out}
    if c["op"] == "decode" and c["append"]:
        res["pools"] = [None, None]
    return res


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    new, total = _lengths(c)
    row, Hkv = c["Hkv"] * D * 2, c["Hkv"]
    if c["op"] == "prompt":
        # (row i of a sequence sees i + 1 keys and those before its first)
        pairs = sum(a * (b - a) + a * (a + 1) // 2 for a, b in zip(new, total))
        return {"bytes": sum(new) * c["Hq"] * D * 4 + sum(total) * 2 * row, "flops": 4 * D * c["Hq"] * pairs}
    if c["op"] == "decode":
        nbytes = sum(total) * 2 * row + c["n"] * c["Hq"] * D * 6 + 4 * sum(_pages_of(x, c["P"]) for x in total)
        if c["append"]:
            nbytes += c["n"] * 4 * row
        return {"bytes": nbytes, "flops": 4 * D * c["Hq"] * sum(total)}
    if c["op"] == "branch":
        held = [_pages_of(x, c["P"]) for x in total]
        # (entries of the table read and written, counts read and written; the rows of half-filled pages)
        books = 4 * sum(6 * k for k in held)
        return {"bytes": books + c["layers"] * sum(x % c["P"] for x in total) * 4 * row, "flops": 0}
    # (the live pages behind the front that holds them all, of a pool in no order)
    pool, live = _pool_pages(c), sum(_pages_of(x, c["P"]) for x in total)
    moved = live * (pool - live) // pool
    return {"bytes": moved * c["P"] * 4 * row + 4 * (pool * 2 + live * 2), "flops": 0}
