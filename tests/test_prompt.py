"""Attention over whole prompts: refusals on the host, and every layout, type and edge against the
definition in 64 bits.

Tolerance of an element y = sum p v / sum p, with A = sum p |v| / sum p and h = finfo(type).eps / 2, half a step:
  h A        each weight is rounded once to the type of V (the sum of weights is of those before it)
  h |y|      the output is rounded once
  2 e A      a logit in binary32 is off by up to e = 130 * 2^-24 * sum |q||k| / sqrt(d) + 2^-20 (128 products summed, two
             more roundings; the exponential): numerator and denominator both move by that share
The largest e of a row's keys serves for the row."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2408_07092_amd as ds

D = 128
FAKE = ctypes.c_void_p(0x10000)   # aligned, never dereferenced: validation fails first
TYPES = {"f16": (torch.float16, ds.DS_F16), "bf16": (torch.bfloat16, ds.DS_BF16)}


# ------------------------------------------------------------------ host
def call(prm, q=FAKE, K=FAKE, V=FAKE, out=FAKE, qs=FAKE, ks=FAKE, kl=FAKE, ws=FAKE, n=1 << 30):
    return ds.lib().ds_prompt_attention(q, K, V, out, qs, ks, kl, ws, n, ctypes.byref(prm) if prm else None, None)


def call_paged(prm, pg, q=FAKE, K=FAKE, V=FAKE, out=FAKE, qs=FAKE, rows=None, lens=FAKE, table=FAKE, ws=FAKE, n=1 << 30):
    return ds.lib().ds_prompt_attention_paged(q, K, V, out, qs, rows, lens, table, ws, n, ctypes.byref(prm) if prm else None,
                                              ctypes.byref(pg) if pg else None, None)


GOOD = dict(n_seqs=3, Hq=8, Hkv=2, d=D, total_q=100, max_kv=50, kv_elems=1 << 20)


def test_refusals():
    ok = ds.prompt(**GOOD)
    for name in ("q", "K", "V", "out", "qs", "ks", "kl", "ws"):
        assert call(ok, **{name: None}) == ds.DS_ERR_NULL, name
    assert call(None) == ds.DS_ERR_NULL
    for bad in (dict(n_seqs=0), dict(total_q=-1), dict(max_kv=-1), dict(Hq=7), dict(Hkv=0), dict(Hq=0), dict(d=64), dict(dtype=2),
                dict(dtype=-1), dict(q_stride=8 * D - 8), dict(q_stride=8 * D + 4), dict(out_stride=4), dict(kv_stride=120),
                dict(kv_stride=D + 1), dict(kv_head_stride=8), dict(kv_elems=-1), dict(kv_stride=(1 << 24) + 8),
                dict(q_stride=-8 * D), dict(kv_head_stride=(1 << 40) + 8), dict(total_q=2**31 - 1), dict(n_seqs=1 << 22)):
        assert call(ds.prompt(**{**GOOD, **bad})) == ds.DS_ERR_SHAPE, bad
        assert ds.ds_prompt_workspace_bytes(ds.prompt(**{**GOOD, **bad})) == 0
    for name in ("q", "K", "V", "out", "ws"):
        assert call(ok, **{name: ctypes.c_void_p(0x10008)}) == ds.DS_ERR_ALIGN, name
    for name in ("qs", "ks", "kl"):
        assert call(ok, **{name: ctypes.c_void_p(0x10002)}) == ds.DS_ERR_ALIGN, name
    need = ds.ds_prompt_workspace_bytes(ok)
    assert need > 0 and need % 256 == 0 and call(ok, n=need - 1) == ds.DS_ERR_WORKSPACE
    assert call(ds.prompt(**{**GOOD, "total_q": 0})) == ds.DS_OK     # no rows: nothing to enqueue


def test_paged_refusals():
    ok, pg = ds.prompt(**GOOD), dict(n_pages=10, page_tokens=16, Hkv=2, d=D, n_rows=3, max_pages=4)
    for name in ("q", "K", "V", "out", "qs", "lens", "table", "ws"):
        assert call_paged(ok, ds.pages(**pg), **{name: None}) == ds.DS_ERR_NULL, name
    assert call_paged(ok, None) == ds.DS_ERR_NULL and call_paged(None, ds.pages(**pg)) == ds.DS_ERR_NULL
    for bad in (dict(page_tokens=8), dict(page_tokens=24), dict(page_tokens=512), dict(page_tokens=0), dict(page_tokens=-16),
                dict(n_pages=0), dict(n_pages=(1 << 20) + 1), dict(Hkv=4), dict(d=64), dict(n_rows=0), dict(n_rows=65537),
                dict(max_pages=0), dict(max_pages=1 << 27), dict(dtype=ds.DS_BF16), dict(dtype=7), dict(n_rows=2)):
        assert call_paged(ok, ds.pages(**{**pg, **bad})) == ds.DS_ERR_SHAPE, bad
    for name in ("K", "V"):
        assert call_paged(ok, ds.pages(**pg), **{name: ctypes.c_void_p(0x10010)}) == ds.DS_ERR_ALIGN, name
    for name in ("qs", "rows", "lens", "table"):
        assert call_paged(ok, ds.pages(**pg), **{name: ctypes.c_void_p(0x10001)}) == ds.DS_ERR_ALIGN, name
    assert call_paged(ok, ds.pages(**pg), n=ds.ds_prompt_workspace_bytes(ok) - 1) == ds.DS_ERR_WORKSPACE


def test_arrays_without_an_element_need_no_address():
    none = ds.prompt(**{**GOOD, "total_q": 0})
    assert call(none, q=None, out=None) == ds.DS_OK and call(ds.prompt(**{**GOOD, "total_q": 0, "kv_elems": 0}), q=None, K=None, V=None, out=None) == ds.DS_OK
    assert call(none, K=None) == ds.DS_ERR_NULL and call(none, q=None, kl=None) == ds.DS_ERR_NULL
    assert call(ds.prompt(**{**GOOD, "total_q": -1}), q=None) == ds.DS_ERR_NULL
    pg = ds.pages(n_pages=10, page_tokens=16, Hkv=2, d=D, n_rows=3, max_pages=4)
    assert call_paged(none, pg, q=None, out=None) == ds.DS_OK and call_paged(none, pg, K=None) == ds.DS_ERR_NULL


# ------------------------------------------------------------------ definition
def defined(q, k, v, before):
    """(y, A, e): q [m, Hq, d], k and v [t, Hkv, d], row i sees the keys up to i + before."""
    m, Hq = q.shape[:2]
    G = Hq // k.shape[1]
    q, k, v = q.double().cpu(), k.double().cpu().repeat_interleave(G, 1), v.double().cpu().repeat_interleave(G, 1)
    s = torch.einsum("mhd,thd->hmt", q, k) / math.sqrt(D)
    size = torch.einsum("mhd,thd->hmt", q.abs(), k.abs()) / math.sqrt(D)
    hidden = torch.arange(k.shape[0])[None, None] > torch.arange(m)[None, :, None] + before
    s = s.masked_fill(hidden, -math.inf)
    p = torch.exp(s - s.amax(2, keepdim=True).clamp(min=-1e300)) if k.shape[0] else s
    total = p.sum(2, keepdim=True).clamp(min=1e-300)
    y = torch.einsum("hmt,thd->mhd", p / total, v)
    A = torch.einsum("hmt,thd->mhd", p / total, v.abs())
    e = size.masked_fill(hidden, 0.0).amax(2) if k.shape[0] else torch.zeros(Hq, m, dtype=torch.double)
    return y, A, (130 * 2.0**-24 * e + 2.0**-20).T[:, :, None]


def near(got, q, k, v, before, dtype):
    y, A, e = defined(q, k, v, before)
    h = torch.finfo(dtype).eps / 2
    tol = h * (A + y.abs()) + 2 * e * A + 1e-7
    off = (got.double().cpu() - y).abs()
    assert torch.isfinite(got).all() and (off <= tol).all(), f"off by {(off / tol).max():.3f} of the tolerance"


def values(shape, dtype, seed, outliers=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    if outliers:
        x[..., ::16] *= 8.0
    return x.to(dtype)


def starts(lengths, first=0):
    return torch.tensor([first] + list(np.cumsum(lengths) + first), dtype=torch.int32)


CANARY = -77.0

# (new tokens of the sequences, keys before them): tile edges (rows of 128 / G tokens, 64 keys), sequences without a token
# and without a key, more new tokens than keys, one token after many
BATCHES = {
    "one_token": ([1], [0]),
    "one_after_many": ([1, 1], [700, 63]),
    "edges": ([63, 64, 65, 128, 129, 1], [0, 0, 0, 0, 0, 0]),
    "empties": ([0, 5, 0, 0, 70, 0], [0, 0, 9, 0, 0, 4]),
    "fewer_keys": ([40, 200, 10], [-7, -130, -10]),
    "parts": ([17, 100, 3, 33], [64, 1000, 127, 31]),
    "long": ([1100], [0]),
}


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(4, 4), (8, 2), (7, 1), (16, 1), (10, 2)], ids=str)
@pytest.mark.parametrize("name", BATCHES)
@pytest.mark.parametrize("dtype", TYPES)
def test_packed_against_definition(dtype, name, heads):
    t, code = TYPES[dtype]
    (Hq, Hkv), (new, before) = heads, BATCHES[name]
    keys = [a + b for a, b in zip(new, before)]
    T, R = sum(new) + 5, sum(keys) + 9
    q, K, V = values((T, Hq, D), t, 1).cuda(), values((R, Hkv, D), t, 2, True).cuda(), values((R, Hkv, D), t, 3).cuda()
    V[sum(keys) + 2:] = math.nan        # behind the last sequence: never part of a result
    K[sum(keys) + 2:] = math.inf
    qs, ks = starts(new, 2), starts(keys, 2)
    out = torch.full((T, Hq, D), CANARY, dtype=t, device="cuda")
    prm = ds.prompt(len(new), Hq, Hkv, D, T, max(keys), code, kv_elems=K.numel())
    ws = ds.ds_prompt_workspace_alloc(prm)
    ds.ds_prompt_attention(q, K, V, out, qs.cuda(), ks[:-1].contiguous().cuda(),
                           torch.tensor(keys, dtype=torch.int32).cuda(), ws, prm)
    torch.cuda.synchronize()
    assert (out[:2] == CANARY).all() and (out[2 + sum(new):] == CANARY).all()
    for i, (m, n, b) in enumerate(zip(new, keys, before)):
        o, r = int(qs[i]), int(ks[i])
        near(out[o:o + m], q[o:o + m], K[r:r + n], V[r:r + n], b, t)
        if b < 0:
            assert (out[o:o - b] == 0).all()      # rows that see no key


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["fused", "cache", "interleaved"])
def test_strided_layouts(layout, dtype):
    t, code = TYPES[dtype]
    Hq, Hkv, new, before = 12, 3, [70, 1, 33], [0, 50, 7] if layout != "fused" else [0, 0, 0]
    keys = [a + b for a, b in zip(new, before)]
    T, qs = sum(new), starts(new)
    wide = values((T, Hq + 2 * Hkv + 1, D), t, 4).cuda()
    out_wide = torch.full((T, Hq + 2, D), CANARY, dtype=t, device="cuda")
    q, out = wide[:, :Hq], out_wide[:, 1:1 + Hq]
    row = wide.stride(0)
    if layout == "fused":
        K, V, ks = wide[:, Hq:Hq + Hkv], wide[:, Hq + Hkv:Hq + 2 * Hkv], qs[:-1]
        more = dict(kv_stride=row, kv_head_stride=D, kv_elems=(T - 1) * row + Hkv * D)
        rows = [(K[a:a + n], V[a:a + n]) for a, n in zip(ks.tolist(), keys)]
    else:
        L_max = max(keys) + 3
        inter = layout == "interleaved"
        kv = torch.full((3, Hkv, L_max, 2, D), math.nan, dtype=t)
        for i, n in enumerate(keys):
            kv[i, :, :n] = values((Hkv, n, 2, D), t, 5 + i)
        kv = kv.cuda()
        K, V = (kv[:, :, :, 0], kv[:, :, :, 1]) if inter else (kv[:, :, :, 0].contiguous(), kv[:, :, :, 1].contiguous())
        step = 2 if inter else 1
        more = dict(kv_stride=D * step, kv_head_stride=L_max * D * step, kv_elems=kv.numel() - D if inter else K.numel())
        ks = torch.arange(3, dtype=torch.int32) * Hkv * L_max
        rows = [(K[i, :, :n].transpose(0, 1), V[i, :, :n].transpose(0, 1)) for i, n in enumerate(keys)]
    prm = ds.prompt(3, Hq, Hkv, D, T, max(keys), code, q_stride=row, out_stride=out_wide.stride(0), **more)
    ws = ds.ds_prompt_workspace_alloc(prm)
    ds.ds_prompt_attention(q, K, V, out, qs.cuda(), ks.contiguous().cuda(), torch.tensor(keys, dtype=torch.int32).cuda(), ws, prm)
    torch.cuda.synchronize()
    assert (out_wide[:, 0] == CANARY).all() and (out_wide[:, -1] == CANARY).all()
    for i, (k, v) in enumerate(rows):
        near(out[int(qs[i]):int(qs[i + 1])], q[int(qs[i]):int(qs[i + 1])], k, v, before[i], t)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("guide", [0, 700, 5000, 200000])
def test_split_keys(guide, dtype):
    """Few rows: the keys are split by the length that is told, whatever the true ones are -- parts with one key, with none
    that a row sees, and none at all -- and joined; a bad place is NaN through the join, and the others are whole."""
    t, code = TYPES[dtype]
    Hq, Hkv, P = 8, 2, 32
    new, before = [3, 1, 0, 20, 2, 65], [4000, 0, 3, -5, 64, 63]
    keys = [a + b for a, b in zip(new, before)]
    T, R = sum(new) + 3, sum(keys)
    q, K, V = values((T, Hq, D), t, 1).cuda(), values((R, Hkv, D), t, 2, True).cuda(), values((R, Hkv, D), t, 3).cuda()
    qs, ks = starts(new, 1), starts(keys)
    prm = ds.prompt(len(new), Hq, Hkv, D, T, guide, code, kv_elems=K.numel())
    ws = ds.ds_prompt_workspace_alloc(prm)
    assert (ws.numel() > 256) == (guide > 0)                    # (there are parts)
    for broken in (False, True):
        lens = torch.tensor(keys, dtype=torch.int32)
        if broken:
            lens[3] = R + 1
        out = torch.full((T, Hq, D), CANARY, dtype=t, device="cuda")
        ds.ds_prompt_attention(q, K, V, out, qs.cuda(), ks[:-1].contiguous().cuda(), lens.cuda(), ws, prm)
        torch.cuda.synchronize()
        assert (out[0] == CANARY).all() and (out[1 + sum(new):] == CANARY).all()
        for i, (m, n, b) in enumerate(zip(new, keys, before)):
            o, r = int(qs[i]), int(ks[i])
            if broken and i == 3:
                assert torch.isnan(out[o:o + m]).all()
                continue
            near(out[o:o + m], q[o:o + m], K[r:r + n], V[r:r + n], b, t)
            if b < 0:
                assert (out[o:o - b] == 0).all()
    Kp, Vp, table, kv = paged(keys, Hkv, P, t, 21)
    rows, lens = torch.arange(1, len(keys) + 1, dtype=torch.int32).cuda(), torch.tensor([9] + keys + [9], dtype=torch.int32).cuda()
    pg = ds.pages(Kp.shape[0], P, Hkv, D, table.shape[0], table.shape[1], code)
    for bad in (None, Kp.shape[0], -1):
        tb = table.clone()
        if bad is not None:
            tb[1, 70] = bad                                     # in the middle of the long one
        out = torch.full((T, Hq, D), CANARY, dtype=t, device="cuda")
        ds.ds_prompt_attention_paged(q, Kp, Vp, out, qs.cuda(), rows, lens, tb, ws, prm, pg)
        torch.cuda.synchronize()
        assert (out[0] == CANARY).all() and (out[1 + sum(new):] == CANARY).all()
        for i, (m, b) in enumerate(zip(new, before)):
            o = int(qs[i])
            if bad is not None and i == 0:
                assert torch.isnan(out[o:o + m]).all()
            else:
                near(out[o:o + m], q[o:o + m], kv[i][0], kv[i][1], b, t)


def paged(keys, Hkv, P, t, seed, spare=3):
    """Pools, table, and the keys and values of the sequences: pages in no order, NaN wherever nobody's rows are."""
    held = [(n + P - 1) // P for n in keys]
    n_pages = sum(held) + spare
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))
    table = torch.full((len(keys) + 2, max(held) + 2), -5, dtype=torch.int32)
    pools = torch.full((2, n_pages, Hkv, P, D), math.nan, dtype=t)
    kv, at = [], 0
    for i, n in enumerate(keys):
        x = values((2, n, Hkv, D), t, seed + 10 + i)
        x[0, ..., ::16] *= 8
        for j in range(held[i]):
            part = x[:, j * P:(j + 1) * P].transpose(1, 2)
            pools[:, order[at], :, :part.shape[2]] = part
            table[i + 1, j] = order[at]
            at += 1
        kv.append(x)
    return pools[0].contiguous().cuda(), pools[1].contiguous().cuda(), table.cuda(), kv


@pytest.mark.gpu
@pytest.mark.parametrize("P", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dtype", TYPES)
def test_paged_against_definition(dtype, P):
    t, code = TYPES[dtype]
    Hq, Hkv = 8, 2
    for name in ("one_after_many", "edges", "empties", "fewer_keys", "parts"):
        new, before = BATCHES[name]
        keys = [a + b for a, b in zip(new, before)]
        Kp, Vp, table, kv = paged(keys, Hkv, P, t, 20)
        T, qs = sum(new) + 1, starts(new)
        q = values((T, Hq, D), t, 1).cuda()
        lens = torch.tensor([999] + keys + [999], dtype=torch.int32).cuda()
        rows = torch.arange(1, len(keys) + 1, dtype=torch.int32).cuda()
        out = torch.full((T, Hq, D), CANARY, dtype=t, device="cuda")
        prm = ds.prompt(len(new), Hq, Hkv, D, T, max(keys), code)
        pg = ds.pages(Kp.shape[0], P, Hkv, D, table.shape[0], table.shape[1], code)
        ws = ds.ds_prompt_workspace_alloc(prm)
        ds.ds_prompt_attention_paged(q, Kp, Vp, out, qs.cuda(), rows, lens, table, ws, prm, pg)
        torch.cuda.synchronize()
        assert (out[-1] == CANARY).all()
        for i, (m, b) in enumerate(zip(new, before)):
            o = int(qs[i])
            near(out[o:o + m], q[o:o + m], kv[i][0], kv[i][1], b, t)


@pytest.mark.gpu
def test_places_that_are_not_there():
    """Sequences whose keys do not lie where they may be read give NaN, those whose rows do not are left alone,
    and the others of the call do not notice."""
    t, code, Hq, Hkv, P, new = torch.float16, ds.DS_F16, 4, 2, 16, [5, 40, 3, 20]
    q = values((sum(new), Hq, D), t, 1).cuda()
    K, V = values((100, Hkv, D), t, 2).cuda(), values((100, Hkv, D), t, 3).cuda()
    qs = starts(new)
    for i, (start, n) in enumerate([(96, 5), (0, 101), (-1, 3), (2**31 - 1, 20)]):   # one row too far, too long, before, far
        ks, kl = [0, 20, 7, 60], [5, 40, 3, 20]
        ks[i], kl[i] = start, n
        out = torch.full((sum(new), Hq, D), CANARY, dtype=t, device="cuda")
        prm = ds.prompt(4, Hq, Hkv, D, sum(new), 101, code, kv_elems=K.numel())
        ds.ds_prompt_attention(q, K, V, out, qs.cuda(), torch.tensor(ks, dtype=torch.int32).cuda(),
                               torch.tensor(kl, dtype=torch.int32).cuda(), ds.ds_prompt_workspace_alloc(prm), prm)
        torch.cuda.synchronize()
        for j in range(4):
            o = slice(int(qs[j]), int(qs[j + 1]))
            if j == i:
                assert torch.isnan(out[o]).all()
            else:
                near(out[o], q[o], K[ks[j]:ks[j] + kl[j]], V[ks[j]:ks[j] + kl[j]], kl[j] - new[j], t)
    # rows of q outside [0, total_q): not computed
    for broken in ([-3, 5, 45, 48, 68], [0, 5, 45, 48, 69], [0, 5, 4, 48, 68]):
        out = torch.full((sum(new), Hq, D), CANARY, dtype=t, device="cuda")
        prm = ds.prompt(4, Hq, Hkv, D, sum(new), 40, code, kv_elems=K.numel())
        ds.ds_prompt_attention(q, K, V, out, torch.tensor(broken, dtype=torch.int32).cuda(),
                               torch.tensor([0, 20, 7, 60], dtype=torch.int32).cuda(), torch.tensor([5, 40, 3, 20], dtype=torch.int32).cuda(),
                               ds.ds_prompt_workspace_alloc(prm), prm)
        torch.cuda.synchronize()
        bad = [i for i in range(4) if not 0 <= broken[i] <= broken[i + 1] <= sum(new)]
        good = [r for i in range(4) if i not in bad for r in range(broken[i], broken[i + 1])]
        left = sorted(set(range(sum(new))) - set(good))
        assert bad and (out[left] == CANARY).all()
    keys = [a + 30 for a in new]
    Kp, Vp, table, kv = paged(keys, Hkv, P, t, 20)
    held = torch.tensor(keys, dtype=torch.int32)
    for i, (row, n, entry) in enumerate([(99, None, None), (None, 2**30, None), (None, None, Kp.shape[0]), (None, None, -1), (-1, None, None), (None, -1, None)]):
        i %= 4
        tb, rows, lens = table.clone(), torch.arange(1, 5, dtype=torch.int32), torch.cat((held[:1], held, held[:1]))
        if row is not None:
            rows[i] = row
        if n is not None:
            lens[i + 1] = n
        if entry is not None:
            tb[i + 1, (keys[i] - 1) // P] = entry
        out = torch.full((sum(new), Hq, D), CANARY, dtype=t, device="cuda")
        prm = ds.prompt(4, Hq, Hkv, D, sum(new), max(keys), code)
        pg = ds.pages(Kp.shape[0], P, Hkv, D, tb.shape[0], tb.shape[1], code)
        ds.ds_prompt_attention_paged(q, Kp, Vp, out, qs.cuda(), rows.cuda(), lens.cuda(), tb, ds.ds_prompt_workspace_alloc(prm), prm, pg)
        torch.cuda.synchronize()
        for j in range(4):
            o = slice(int(qs[j]), int(qs[j + 1]))
            if j == i:
                assert torch.isnan(out[o]).any(dim=(1, 2)).any()
                assert row is None and n is None or torch.isnan(out[o]).all()
            else:
                near(out[o], q[o], kv[j][0], kv[j][1], 30, t)


@pytest.mark.gpu
def test_extreme_weights():
    """Logits far apart, a maximum that rises late and by little and by much, and equal logits over many keys."""
    for t, code in TYPES.values():
        q = torch.zeros((40, 2, D), dtype=t)
        q[:, :, 0] = 30.0
        K, V = torch.zeros((600, 1, D), dtype=t), values((600, 1, D), t, 3)
        K[:, 0, 0] = torch.cat((torch.linspace(-200, 0, 300), torch.linspace(0, 3, 150), torch.full((100,), 3.0), torch.linspace(3, 200, 50))).to(t)
        q[1::2, 1, 0] = 0.0
        qs, kl = starts([40]), torch.tensor([600], dtype=torch.int32)
        out = torch.zeros_like(q).cuda()
        prm = ds.prompt(1, 2, 1, D, 40, 600, code, kv_elems=K.numel())
        ds.ds_prompt_attention(q.cuda(), K.cuda(), V.cuda(), out, qs.cuda(), torch.zeros(1, dtype=torch.int32).cuda(), kl.cuda(),
                               ds.ds_prompt_workspace_alloc(prm), prm)
        torch.cuda.synchronize()
        near(out, q, K, V, 560, t)


@pytest.mark.gpu
@pytest.mark.parametrize("guide", [0, 60000])
@pytest.mark.parametrize("form", ["packed", "paged"])
@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_not_seen_is_not_finite(dtype, form, guide):
    """Values and keys that are infinite or NaN touch the rows that see them, and there the channels that they are in:
    not the rows before them, which share their tiles, nor other heads or sequences."""
    t, code = TYPES[dtype]
    Hq, Hkv, P, new, before = 6, 2, 16, [150, 20], [0, 300]
    keys = [a + b for a, b in zip(new, before)]
    qs, q = starts(new), values((sum(new), Hq, D), t, 1)
    kv = [values((2, n, Hkv, D), t, 40 + i) for i, n in enumerate(keys)]
    broken = [x.clone() for x in kv]
    broken[0][1, 100, 0, 5], broken[0][1, 120, 0, 7] = math.inf, -math.inf     # values of KV head 0: rows 100.., 120..
    broken[0][1, 149, 1, :] = math.nan                                         # of head 1: the last row alone
    broken[1][0, 310, 1, 9] = math.nan                                         # a key of head 1, of the other sequence
    prm = ds.prompt(2, Hq, Hkv, D, sum(new), guide, code, kv_elems=sum(keys) * Hkv * D)
    ws = ds.ds_prompt_workspace_alloc(prm)
    assert (ws.numel() > 256) == (guide > 0)
    out = torch.full((sum(new), Hq, D), CANARY, dtype=t, device="cuda")
    if form == "packed":
        K, V = (torch.cat([x[i] for x in broken]).cuda() for i in (0, 1))
        ds.ds_prompt_attention(q.cuda(), K, V, out, qs.cuda(), starts(keys)[:-1].contiguous().cuda(),
                               torch.tensor(keys, dtype=torch.int32).cuda(), ws, prm)
    else:
        Kp, Vp, table, _ = paged(keys, Hkv, P, t, 20)
        for i, x in enumerate(broken):
            for j in range(keys[i]):
                p = int(table[i + 1, j // P])
                Kp[p, :, j % P], Vp[p, :, j % P] = x[0, j].cuda(), x[1, j].cuda()
        pg = ds.pages(Kp.shape[0], P, Hkv, D, table.shape[0], table.shape[1], code)
        ds.ds_prompt_attention_paged(q.cuda(), Kp, Vp, out, qs.cuda(), torch.tensor([1, 2], dtype=torch.int32).cuda(),
                                     torch.tensor([0] + keys + [0], dtype=torch.int32).cuda(), table, ws, prm, pg)
    torch.cuda.synchronize()
    got, G = out.cpu(), Hq // Hkv
    touched = torch.zeros(got.shape, dtype=torch.bool)
    touched[100:150, :G, 5] = touched[120:150, :G, 7] = touched[149, G:] = touched[160:, G:] = True
    assert not torch.isfinite(got[touched]).any()
    for i, (m, b) in enumerate(zip(new, before)):
        o = slice(int(qs[i]), int(qs[i + 1]))
        y, A, e = defined(q[o], kv[i][0], kv[i][1], b)
        # (a channel of a row that sees an infinity elsewhere: as if the infinity were any number there)
        tol = torch.finfo(t).eps / 2 * (A + y.abs()) + 2 * e * A + 1e-7
        assert ((got[o].double() - y).abs() <= tol)[~touched[o]].all()


@pytest.mark.gpu
@pytest.mark.parametrize("guide", [0, 60000])
@pytest.mark.parametrize("dtype", TYPES)
def test_scores_of_minus_infinity(dtype, guide):
    """A key whose score is -infinity has no weight; a row of them alone is 0 / 0."""
    t, code = TYPES[dtype]
    q, K, V = values((200, 2, D), t, 1), values((200, 1, D), t, 2), values((200, 1, D), t, 3)
    q[:, :, 0] = 1.0
    K[:70, :, 0] = -math.inf
    prm = ds.prompt(1, 2, 1, D, 200, guide, code, kv_elems=K.numel())
    ws, zero, n = ds.ds_prompt_workspace_alloc(prm), torch.zeros(1, dtype=torch.int32).cuda(), torch.tensor([200], dtype=torch.int32).cuda()
    out = torch.zeros_like(q).cuda()
    ds.ds_prompt_attention(q.cuda(), K.cuda(), V.cuda(), out, starts([200]).cuda(), zero, n, ws, prm)
    torch.cuda.synchronize()
    assert torch.isnan(out[:70]).all()
    near(out[70:], q[70:], K[70:], V[70:], 0, t)


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(64, 64), (96, 32)], ids=str)
def test_more_workgroups_than_compute_units_but_not_twice_as_many(heads):
    """Every row tile of every head has its workgroup where they are dealt out by weight."""
    t, code, (Hq, Hkv), new = torch.bfloat16, ds.DS_BF16, heads, [300, 220]
    tiles = sum(new) * (Hq // Hkv) // 128 + len(new)
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    assert cus < tiles * Hkv <= 2 * cus
    T, qs = sum(new), starts(new)
    q, K, V = values((T, Hq, D), t, 1).cuda(), values((T, Hkv, D), t, 2, True).cuda(), values((T, Hkv, D), t, 3).cuda()
    prm = ds.prompt(2, Hq, Hkv, D, T, max(new), code, kv_elems=K.numel())
    out = torch.full((T, Hq, D), CANARY, dtype=t, device="cuda")
    ds.ds_prompt_attention(q, K, V, out, qs.cuda(), qs[:-1].contiguous().cuda(), torch.tensor(new, dtype=torch.int32).cuda(),
                           ds.ds_prompt_workspace_alloc(prm), prm)
    torch.cuda.synchronize()
    for i in range(2):
        r = slice(int(qs[i]), int(qs[i + 1]))
        near(out[r], q[r], K[r], V[r], 0, t)


@pytest.mark.gpu
@pytest.mark.parametrize("guide", [0, 600])
@pytest.mark.parametrize("form", ["packed", "paged"])
@pytest.mark.parametrize("dtype", TYPES)
def test_few_tiles_of_many_heads(dtype, form, guide):
    """One to four tiles of keys, two workgroups to a compute unit, wavefronts of unlike work in a workgroup (down to one tile of
    three): the first tile is whole until all of them have read it.  Again and again the same bits, the definition's."""
    t, code, P = TYPES[dtype] + (16,)
    Hq = Hkv = 96
    new, before = [97, 128, 128, 100, 128, 65, 70], [0, 1, 32, 17, 60, 130, 0]
    if guide:      # fewer rows, so that the keys are split; parts of up to three tiles
        Hq = Hkv = 8
        new, before = [97, 128, 70], [400, 501, 32]
    keys = [a + b for a, b in zip(new, before)]
    T, qs, ks = sum(new), starts(new), starts(keys)
    q = values((T, Hq, D), t, 1).cuda()
    Kp, Vp, table, kv = paged(keys, Hkv, P, t, 50)
    K, V = (torch.cat([x[i] for x in kv]).cuda() for i in (0, 1))
    rows, lens = torch.arange(1, len(keys) + 1, dtype=torch.int32).cuda(), torch.tensor([9] + keys + [9], dtype=torch.int32).cuda()
    prm = ds.prompt(len(new), Hq, Hkv, D, T, guide, code, kv_elems=K.numel())
    pg = ds.pages(Kp.shape[0], P, Hkv, D, table.shape[0], table.shape[1], code)
    ws = ds.ds_prompt_workspace_alloc(prm)
    assert (ws.numel() > 256) == (guide > 0)
    args = qs.cuda(), ks[:-1].contiguous().cuda(), torch.tensor(keys, dtype=torch.int32).cuda()
    first = None
    for _ in range(30):
        out = torch.full((T, Hq, D), CANARY, dtype=t, device="cuda")
        if form == "packed":
            ds.ds_prompt_attention(q, K, V, out, *args, ws, prm)
        else:
            ds.ds_prompt_attention_paged(q, Kp, Vp, out, args[0], rows, lens, table, ws, prm, pg)
        torch.cuda.synchronize()
        if first is None:
            first = out
            for i, (m, b) in enumerate(zip(new, before)):
                o = slice(int(qs[i]), int(qs[i + 1]))
                near(out[o], q[o], kv[i][0], kv[i][1], b, t)
        assert torch.equal(out, first)


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["packed", "paged", "split"])
@pytest.mark.parametrize("size", [3e33, 1e34, 1e35, 3.3895e38])
def test_over_the_range_of_bf16(size, form):
    """Values as large as bf16 has, equal ones that add up among them, within a part of split keys and over the parts: the result is a
    number, theirs."""
    t, code, P, Hq, Hkv, new, before = torch.bfloat16, ds.DS_BF16, 32, 6, 2, [1, 70, 300, 40], [0, 0, 63, 1000]
    if form == "split":
        new, before = [3, 20, 1], [1000, 4000, 64]
    keys = [a + b for a, b in zip(new, before)]
    T, qs, ks = sum(new), starts(new), starts(keys)
    Kp, Vp, table, kv = paged(keys, Hkv, P, t, 51)
    for i, x in enumerate(kv):
        v = x[1].float()
        x[1] = torch.where(torch.arange(D) % 3 == 0, torch.full_like(v, size), v / v.abs().max() * size).to(t)
        assert torch.isfinite(x[1]).all()
        for j in range((keys[i] + P - 1) // P):
            part = x[1, j * P:(j + 1) * P].transpose(0, 1)
            Vp[table[i + 1, j], :, :part.shape[1]] = part.cuda()
    q = values((T, Hq, D), t, 1)
    q[:, 0] = 0.0                                  # (equal weights)
    K, V = (torch.cat([x[i] for x in kv]).cuda() for i in (0, 1))
    out = torch.full((T, Hq, D), CANARY, dtype=t, device="cuda")
    prm = ds.prompt(len(new), Hq, Hkv, D, T, 60000 if form == "split" else 0, code, kv_elems=K.numel())
    assert (ds.ds_prompt_workspace_bytes(prm) > 256) == (form == "split")
    if form != "paged":
        ds.ds_prompt_attention(q.cuda(), K, V, out, qs.cuda(), ks[:-1].contiguous().cuda(), torch.tensor(keys, dtype=torch.int32).cuda(),
                               ds.ds_prompt_workspace_alloc(prm), prm)
    else:
        pg = ds.pages(Kp.shape[0], P, Hkv, D, table.shape[0], table.shape[1], code)
        ds.ds_prompt_attention_paged(q.cuda(), Kp, Vp, out, qs.cuda(), torch.arange(1, len(keys) + 1, dtype=torch.int32).cuda(),
                                     torch.tensor([9] + keys + [9], dtype=torch.int32).cuda(), table, ds.ds_prompt_workspace_alloc(prm), prm, pg)
    torch.cuda.synchronize()
    for i, (m, b) in enumerate(zip(new, before)):
        o = slice(int(qs[i]), int(qs[i + 1]))
        near(out[o].double().cpu() / size, q[o], kv[i][0], kv[i][1].double() / size, b, t)


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["packed", "paged"])
@pytest.mark.parametrize("what", ["first_value", "all_values", "first_key", "queries"])
def test_cost_of_what_is_not_finite(what, form):
    """A NaN that all rows of a prompt see, values of which none is finite (each row has hidden ones in its tiles), rows of q that are NaN: all
    rows are formed twice, which costs a small factor and does not grow with the length as the rows themselves do."""
    t, code, P, Hq, Hkv, n = torch.float16, ds.DS_F16, 64, 16, 8, 4096
    q, K, V = values((n, Hq, D), t, 1).cuda(), values((n, Hkv, D), t, 2).cuda(), values((n, Hkv, D), t, 3).cuda()
    {"first_value": V[0], "all_values": V, "first_key": K[0], "queries": q}[what][..., 5] = math.nan
    good = values((n, Hkv, D), t, 3).cuda(), values((n, Hkv, D), t, 2).cuda(), values((n, Hq, D), t, 1).cuda()
    out = torch.empty_like(q)
    prm = ds.prompt(1, Hq, Hkv, D, n, n, code, kv_elems=K.numel())
    ws, zero, ends, length = ds.ds_prompt_workspace_alloc(prm), ints_([0]), ints_([0, n]), ints_([n])
    table = torch.arange(n // P, dtype=torch.int32, device="cuda")[None]
    pg = ds.pages(n // P, P, Hkv, D, 1, n // P, code)
    pools = lambda x: x.reshape(n // P, P, Hkv, D).transpose(1, 2).contiguous()  # noqa: E731

    def passes(q, K, V):
        if form == "paged":
            K, V = pools(K), pools(V)
            run = lambda: ds.ds_prompt_attention_paged(q, K, V, out, ends, None, length, table, ws, prm, pg)  # noqa: E731
        else:
            run = lambda: ds.ds_prompt_attention(q, K, V, out, ends, zero, length, ws, prm)  # noqa: E731
        run()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda.synchronize()
        a.record()
        for _ in range(5):
            run()
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b) / 5

    plain, strange = passes(good[2], good[1], good[0]), passes(q, K, V)
    print(f"{what} {form}: {1000 * plain:.0f} -> {1000 * strange:.0f} us")
    touched = torch.isnan(out).any(dim=1)
    assert touched[:, 5].all() and (what not in ("first_value", "all_values") or not torch.isnan(out[..., :5]).any())
    assert strange < 20 * plain


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["packed", "paged"])
def test_a_workspace_of_another_prompt(form):
    """That of a long prompt, which is the least that there is, serves a short part over many keys, and so does any size between that and
    the part's own: with fewer parts, within its bytes."""
    t, code, P, Hq, Hkv, new, before = torch.float16, ds.DS_F16, 16, 8, 2, [3, 16], [2000, 5000]
    keys = [a + b for a, b in zip(new, before)]
    T, qs, ks = sum(new), starts(new), starts(keys)
    Kp, Vp, table, kv = paged(keys, Hkv, P, t, 52)
    q, K, V = values((T, Hq, D), t, 1).cuda(), torch.cat([x[0] for x in kv]).cuda(), torch.cat([x[1] for x in kv]).cuda()
    prm = ds.prompt(2, Hq, Hkv, D, T, max(keys), code, kv_elems=K.numel())
    pg = ds.pages(Kp.shape[0], P, Hkv, D, table.shape[0], table.shape[1], code)
    long = ds.ds_prompt_workspace_bytes(ds.prompt(1, Hq, Hkv, D, 8192, 8192, code, kv_elems=K.numel()))
    need = ds.ds_prompt_workspace_bytes(prm)
    assert long == 256 and need > 8 * T * Hq * 520
    for size in (long, 2 * T * Hq * 520, 3 * T * Hq * 520 + 255, need - 1, need, need + 999):
        ws = torch.full((size + 64,), 0x5a, dtype=torch.uint8, device="cuda")
        out = torch.full((T, Hq, D), CANARY, dtype=t, device="cuda")
        if form == "packed":
            ds.ds_prompt_attention(q, K, V, out, qs.cuda(), ks[:-1].contiguous().cuda(), ints_(keys), ws[:size], prm)
        else:
            ds.ds_prompt_attention_paged(q, Kp, Vp, out, qs.cuda(), ints_([1, 2]), ints_([9] + keys + [9]), table, ws[:size], prm, pg)
        torch.cuda.synchronize()
        assert (ws[size:] == 0x5a).all()
        for i, (m, b) in enumerate(zip(new, before)):
            o = slice(int(qs[i]), int(qs[i + 1]))
            near(out[o], q[o], kv[i][0], kv[i][1], b, t)


@pytest.mark.gpu
@pytest.mark.parametrize("guide", [0, 60000])
@pytest.mark.parametrize("heads", [(8, 2), (2, 2), (6, 1)], ids=str)
def test_which_rows_a_missing_page_makes_nan(heads, guide):
    """Those of the row tiles whose key tiles reach it: every row that sees it, none of the tiles before."""
    t, code, P, (Hq, Hkv), new, before = torch.float16, ds.DS_F16, 16, heads, [3, 300, 40], [20, 41, 0]
    G, keys = Hq // Hkv, [a + b for a, b in zip(new, before)]
    T, qs = sum(new), starts(new)
    if guide:
        new, T, qs = [3, 100, 40], 143, starts([3, 100, 40])
        before = [20, 241, 0]
    Kp, Vp, table, kv = paged(keys, Hkv, P, t, 53)
    q, rows, lens = values((T, Hq, D), t, 1).cuda(), ints_([1, 2, 3]), ints_([9] + keys + [9])
    prm = ds.prompt(3, Hq, Hkv, D, T, guide, code)
    pg = ds.pages(Kp.shape[0], P, Hkv, D, table.shape[0], table.shape[1], code)
    ws = ds.ds_prompt_workspace_alloc(prm)
    assert (ws.numel() > 256) == (guide > 0)
    for page in (0, 2, 5, 12, 17, 21):
        tb = table.clone()
        tb[2, page] = (Kp.shape[0], -1)[page % 2]
        out = torch.full((T, Hq, D), CANARY, dtype=t, device="cuda")
        ds.ds_prompt_attention_paged(q, Kp, Vp, out, qs.cuda(), rows, lens, tb, ws, prm, pg)
        torch.cuda.synchronize()
        want = torch.zeros((new[1], Hkv, G), dtype=torch.bool)
        for i in range(new[1]):
            for g in range(G):
                last = (min((i * G + g) // 128 * 128 + 128, new[1] * G) - 1) // G           # the tile's last token
                reach = min(keys[1], (last + before[1] + 64) // 64 * 64)
                want[i, :, g] = page * P < reach
                assert want[i, 0, g] or page * P > i + before[1]
        mine = out[int(qs[1]):int(qs[2])].cpu()
        want = want.reshape(new[1], Hq)
        assert torch.equal(torch.isnan(mine).any(dim=2), want) and torch.equal(torch.isnan(mine).all(dim=2), want)
        free = int((~want.any(dim=1)).sum())                                                # (rows of the tiles before come first)
        near(mine[:free], q[int(qs[1]):int(qs[1]) + free], kv[1][0][:free + before[1]], kv[1][1][:free + before[1]], before[1], t)
        for i in (0, 2):
            o = slice(int(qs[i]), int(qs[i + 1]))
            near(out[o], q[o], kv[i][0], kv[i][1], before[i], t)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_no_rows_and_no_keys(dtype):
    """Empty tensors, which have no address: no new tokens is nothing to do, no keys is rows of zeros."""
    t, code = TYPES[dtype]
    for rows, guide in ((0, 0), (40, 0), (3, 30000)):
        q, K, out = values((rows, 4, D), t, 1).cuda(), torch.empty((0, 2, D), dtype=t, device="cuda"), torch.full((rows, 4, D), CANARY, dtype=t, device="cuda")
        prm = ds.prompt(2, 4, 2, D, rows, guide, code)
        ds.ds_prompt_attention(q, K, K, out, ints_([0, rows // 3, rows]), ints_([0, 0]), ints_([0, 0]), ds.ds_prompt_workspace_alloc(prm), prm)
        assert (out == 0).all()
    pg = ds.pages(1, 16, 2, D, 1, 1, code)
    pool = torch.full((1, 2, 16, D), 3.0, dtype=t, device="cuda")
    ds.ds_append_paged(K, K, pool, pool, ints_([0, 0]), None, ints_([0]), ints_([[0]]), pg, 1)
    assert (pool == 3.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(20, 1), (40, 2), (64, 1), (200, 1)], ids=str)
@pytest.mark.parametrize("dtype", TYPES)
def test_groups_of_more_than_16_heads(dtype, heads):
    """... up to more heads in a group than a row tile has rows."""
    t, code, (Hq, Hkv), new, before = *TYPES[dtype], heads, [1, 70, 33], [5, 0, 100]
    keys = [a + b for a, b in zip(new, before)]
    T, qs, ks = sum(new), starts(new), starts(keys)
    q, K, V = values((T, Hq, D), t, 1).cuda(), values((sum(keys), Hkv, D), t, 2, True).cuda(), values((sum(keys), Hkv, D), t, 3).cuda()
    out = torch.full((T, Hq, D), CANARY, dtype=t, device="cuda")
    prm = ds.prompt(3, Hq, Hkv, D, T, max(keys), code, kv_elems=K.numel())
    ds.ds_prompt_attention(q, K, V, out, qs.cuda(), ks[:-1].contiguous().cuda(), ints_(keys), ds.ds_prompt_workspace_alloc(prm), prm)
    for i, (m, n, b) in enumerate(zip(new, keys, before)):
        o, r = int(qs[i]), int(ks[i])
        near(out[o:o + m], q[o:o + m], K[r:r + n], V[r:r + n], b, t)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_long_prompts(dtype):
    """Many tiles ahead of the causal edge, with heads alone and in pairs."""
    t, code = TYPES[dtype]
    for Hq, Hkv, new, before in ((2, 2, [5003], [0]), (2, 1, [3000, 1200], [1100, 4000])):
        keys = [a + b for a, b in zip(new, before)]
        T, qs, ks = sum(new), starts(new), starts(keys)
        q, K, V = values((T, Hq, D), t, 1).cuda(), values((sum(keys), Hkv, D), t, 2, True).cuda(), values((sum(keys), Hkv, D), t, 3).cuda()
        out = torch.full((T, Hq, D), CANARY, dtype=t, device="cuda")
        prm = ds.prompt(len(new), Hq, Hkv, D, T, max(keys), code, kv_elems=K.numel())
        ds.ds_prompt_attention(q, K, V, out, qs.cuda(), ks[:-1].contiguous().cuda(), ints_(keys), ds.ds_prompt_workspace_alloc(prm), prm)
        for i, (m, n, b) in enumerate(zip(new, keys, before)):
            o, r = int(qs[i]), int(ks[i])
            near(out[o:o + m], q[o:o + m], K[r:r + n], V[r:r + n], b, t)


@pytest.mark.gpu
def test_caches_beyond_32_bit_offsets():
    """Contiguous caches of more than 2^32 elements: the last head of the last entry, as of the first, split and whole."""
    t, Hq, Hkv, L_max, n = torch.float16, 16, 8, 2_200_000, 400
    K, V = (torch.empty((2, Hkv, L_max, D), dtype=t, device="cuda") for _ in range(2))
    assert K.numel() > 1 << 32
    rows = values((2, 2, Hkv, n, D), t, 4).cuda()
    for b in range(2):
        K[b, :, :n], V[b, :, :n] = rows[b, 0], rows[b, 1]
    q, out = values((200, Hq, D), t, 1).cuda(), torch.empty((200, Hq, D), dtype=t, device="cuda")
    for guide in (0, 5000):
        prm = ds.prompt(2, Hq, Hkv, D, 200, guide, ds.DS_F16, kv_stride=D, kv_head_stride=L_max * D, kv_elems=K.numel())
        ws = ds.ds_prompt_workspace_alloc(prm)
        assert (ws.numel() > 256) == (guide > 0)
        ds.ds_prompt_attention(q, K, V, out.fill_(CANARY), ints_([0, 100, 200]), ints_([0, Hkv * L_max]), ints_([n, n]), ws, prm)
        for b in range(2):
            near(out[100 * b:100 * b + 100], q[100 * b:100 * b + 100], rows[b, 0].transpose(0, 1), rows[b, 1].transpose(0, 1), n - 100, t)


def ints_(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")
