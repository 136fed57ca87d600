"""Attention of one new token over a paged cache and the writing of its pages' rows: refusals on the host, and
lengths, pages, heads and types against the definition in 64 bits.

Tolerance of an element y = sum p v / sum p over n tokens, with A = sum p |v| / sum p and h = finfo(type).eps / 2:
  h^2 A                  a weight is the sum of two numbers of V's type, the second the rounded rest of the first
  2 e A                  a logit is off by up to e = 130 * 2^-24 * sum |q||k| / sqrt(d) + 2^-20 (see test_prompt.py)
  2 (n/4 + 300) 2^-24 A  sums in binary32: a wavefront adds every fourth 16 tokens, then states and parts are joined;
                         numerator and denominator"""
import ctypes
import math

import pytest
import torch

import paper_2408_07092_amd as ds
from test_prompt import CANARY, D, FAKE, TYPES, defined, paged, values


# ------------------------------------------------------------------ host
PG = dict(n_pages=10, page_tokens=16, Hkv=2, d=D, n_rows=3, max_pages=4)


def decode(pg, n=3, Hq=4, max_len=60, q=FAKE, K=FAKE, V=FAKE, out=FAKE, rows=None, lens=FAKE, table=FAKE, ws=FAKE, nbytes=1 << 30):
    return ds.lib().ds_paged_decode(q, K, V, out, rows, lens, table, ws, nbytes, ctypes.byref(pg) if pg else None, n, Hq, max_len, None)


def append(pg, n=3, total=5, stride=0, k=FAKE, v=FAKE, K=FAKE, V=FAKE, new_start=FAKE, rows=None, start=FAKE, table=FAKE):
    return ds.lib().ds_append_paged(k, v, K, V, new_start, rows, start, table, ctypes.byref(pg) if pg else None, n, total, stride, None)


BAD_PAGES = (dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=512), dict(n_pages=0), dict(n_pages=(1 << 20) + 1),
             dict(Hkv=0), dict(Hkv=-2), dict(d=64), dict(n_rows=0), dict(n_rows=65537), dict(max_pages=0), dict(max_pages=1 << 27),
             dict(dtype=2), dict(dtype=-1))
OFF = {16: ctypes.c_void_p(0x10008), 256: ctypes.c_void_p(0x10010), 4: ctypes.c_void_p(0x10002)}


def test_decode_refusals():
    ok = ds.pages(**PG)
    for name in ("q", "K", "V", "out", "lens", "table", "ws"):
        assert decode(ok, **{name: None}) == ds.DS_ERR_NULL, name
    assert decode(None) == ds.DS_ERR_NULL
    for bad in BAD_PAGES:
        assert decode(ds.pages(**{**PG, **bad})) == ds.DS_ERR_SHAPE, bad
        assert ds.ds_paged_workspace_bytes(ds.pages(**{**PG, **bad}), 3, 4, 60) == 0
    for bad in (dict(n=0), dict(Hq=3), dict(Hq=0), dict(max_len=-1), dict(n=4)):   # (four sequences, three rows, no list of rows)
        assert decode(ok, **bad) == ds.DS_ERR_SHAPE, bad
    assert decode(ds.pages(**{**PG, "max_pages": 1 << 26}), n=3, Hq=704) == ds.DS_ERR_SHAPE   # 3 * 2 * 22 units of 2^24 pieces: beyond 2^31
    for name, by in (("q", 16), ("out", 16), ("ws", 16), ("K", 256), ("V", 256), ("rows", 4), ("lens", 4), ("table", 4)):
        assert decode(ok, **{name: OFF[by]}) == ds.DS_ERR_ALIGN, name
    need = ds.ds_paged_workspace_bytes(ok, 3, 4, 60)
    assert need > 0 and need % 256 == 0 and decode(ok, nbytes=need - 1) == ds.DS_ERR_WORKSPACE
    assert ds.lib().ds_paged_workspace_bytes(None, 3, 4, 60) == 0


def test_append_refusals():
    ok = ds.pages(**PG)
    for name in ("k", "v", "K", "V", "new_start", "start", "table"):
        assert append(ok, **{name: None}) == ds.DS_ERR_NULL, name
    assert append(None) == ds.DS_ERR_NULL
    for bad in BAD_PAGES:
        assert append(ds.pages(**{**PG, **bad})) == ds.DS_ERR_SHAPE, bad
    for bad in (dict(n=0), dict(n=4), dict(total=-1), dict(stride=2 * D - 8), dict(stride=2 * D + 4), dict(stride=-2 * D),
                dict(total=(1 << 26) + 1), dict(stride=(1 << 30) + 8)):
        assert append(ok, **bad) == ds.DS_ERR_SHAPE, bad
    for name, by in (("k", 16), ("v", 16), ("K", 256), ("V", 256), ("new_start", 4), ("rows", 4), ("start", 4), ("table", 4)):
        assert append(ok, **{name: OFF[by]}) == ds.DS_ERR_ALIGN, name
    assert append(ok, total=0) == ds.DS_OK


def test_append_refuses_what_no_launch_holds():
    """Wavefronts in fours: the last three counts below 2^26 would fill a launch of 2^32 threads."""
    for Hkv, parts in ((2, 1), (8, 1), (9, 2), (128, 16)):
        pg = ds.pages(**{**PG, "Hkv": Hkv})
        for total in (((1 << 26) - 4) // parts + 1, ((1 << 26) - 1) // parts):
            assert total * parts <= (1 << 26) - 4 or append(pg, total=total) == ds.DS_ERR_SHAPE, (Hkv, total)


# ------------------------------------------------------------------ decode
def near(got, q, k, v, dtype):
    n = k.shape[0]
    y, A, e = defined(q[None], k, v, n - 1)
    h = torch.finfo(dtype).eps / 2
    tol = ((h * h + 2 * e + 2 * (n / 4 + 300) * 2.0**-24) * A + 1e-7)[0]
    off = (got.double().cpu() - y[0]).abs()
    assert torch.isfinite(got).all() and (off <= tol).all(), f"off by {(off / tol).max():.3f} of the tolerance"


LENGTHS = {
    "one": [1],
    "short": [1, 15, 16, 17, 63, 64, 65, 127, 128, 129],
    "ragged": [0, 3000, 1, 0, 0, 257, 40, 0],
    "many": [(i * 37) % 90 for i in range(300)],      # more sequences than threads of a workgroup
    "long": [20011, 5],
}


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(2, 2), (6, 2), (7, 1), (12, 1), (16, 1), (40, 2)], ids=str)   # groups of 1, 3, 7, 12, 16, 20
@pytest.mark.parametrize("name", LENGTHS)
@pytest.mark.parametrize("dtype", TYPES)
def test_decode_against_definition(dtype, name, heads):
    t, code = TYPES[dtype]
    (Hq, Hkv), keys = heads, LENGTHS[name]
    P = {"one": 16, "short": 32, "ragged": 16, "many": 64, "long": 128}[name]
    Kp, Vp, table, kv = paged(keys, Hkv, P, t, 30)
    q = values((len(keys), Hq, D), t, 1).cuda()
    lens = torch.tensor([7] + keys + [7], dtype=torch.int32).cuda()
    rows = torch.arange(1, len(keys) + 1, dtype=torch.int32).cuda()
    out = torch.full((len(keys) + 2, Hq, D), CANARY, device="cuda")
    pg = ds.pages(Kp.shape[0], P, Hkv, D, table.shape[0], table.shape[1], code)
    ws = ds.ds_paged_workspace_alloc(pg, len(keys), Hq, max(keys))
    for _ in range(2):       # (counters are zero again after a call)
        ds.ds_paged_decode(q, Kp, Vp, out[1:-1], rows, lens, table, ws, pg, len(keys), Hq, max(keys))
    torch.cuda.synchronize()
    assert (out[0] == CANARY).all() and (out[-1] == CANARY).all()
    for i, n in enumerate(keys):
        if n == 0:
            assert (out[i + 1] == 0).all()
        else:
            near(out[i + 1], q[i], kv[i][0], kv[i][1], t)


@pytest.mark.gpu
@pytest.mark.parametrize("P", [16, 32, 64, 128, 256])
def test_decode_page_sizes_and_a_wrong_guide(P):
    """Pages of every size; a length to plan for that is far below or above the true ones changes no more than bits."""
    t, code, keys, Hq, Hkv = torch.bfloat16, ds.DS_BF16, [P - 1, P, P + 1, 5 * P + 3, 1], 8, 2
    Kp, Vp, table, kv = paged(keys, Hkv, P, t, 31)
    table, lens = table[1:-1].contiguous(), torch.tensor(keys, dtype=torch.int32).cuda()
    q = values((len(keys), Hq, D), t, 1).cuda()
    pg = ds.pages(Kp.shape[0], P, Hkv, D, table.shape[0], table.shape[1], code)
    for guide in (0, max(keys), 100 * max(keys)):
        out = torch.full((len(keys), Hq, D), CANARY, device="cuda")
        ds.ds_paged_decode(q, Kp, Vp, out, None, lens, table, ds.ds_paged_workspace_alloc(pg, len(keys), Hq, guide), pg, len(keys), Hq, guide)
        torch.cuda.synchronize()
        for i in range(len(keys)):
            near(out[i], q[i], kv[i][0], kv[i][1], t)


@pytest.mark.gpu
def test_decode_places_that_are_not_there():
    """A row, a length or a page that cannot be: NaN for that sequence, nothing else changes and nothing stays behind
    in the workspace."""
    t, code, P, Hq, Hkv, keys = torch.float16, ds.DS_F16, 16, 4, 2, [40, 700, 3, 90]
    Kp, Vp, table, kv = paged(keys, Hkv, P, t, 32)
    q = values((4, Hq, D), t, 1).cuda()
    pg = ds.pages(Kp.shape[0], P, Hkv, D, table.shape[0], table.shape[1], code)
    ws = ds.ds_paged_workspace_alloc(pg, 4, Hq, 700)
    good_rows, good_lens = torch.arange(1, 5, dtype=torch.int32), torch.tensor([1] + keys + [1], dtype=torch.int32)
    for i, what in enumerate(("row", "before", "long", "page", "row_far", "negative", "page_before", "none")):
        i %= 4
        rows, lens, tb = good_rows.clone(), good_lens.clone(), table.clone()
        if what in ("row", "row_far", "before"):
            rows[i] = {"row": table.shape[0], "row_far": 2**31 - 1, "before": -1}[what]
        if what in ("long", "negative"):
            lens[i + 1] = {"long": table.shape[1] * P + 1, "negative": -5}[what]
        if what in ("page", "page_before"):
            tb[i + 1, (keys[i] - 1) // P // 2] = {"page": Kp.shape[0], "page_before": -1}[what]
        out = torch.full((4, Hq, D), CANARY, device="cuda")
        ds.ds_paged_decode(q, Kp, Vp, out, rows.cuda(), lens.cuda(), tb, ws, pg, 4, Hq, 700)
        torch.cuda.synchronize()
        for j in range(4):
            if j == i and what != "none":
                assert torch.isnan(out[j]).all(), what
            else:
                near(out[j], q[j], kv[j][0], kv[j][1], t)


@pytest.mark.gpu
def test_decode_beyond_32_bit_offsets():
    """A pool of more than 4 GiB: pages at its far end are reached, by the decode, the prompt and the writing."""
    t, code, P, Hkv, Hq, n = torch.float16, ds.DS_F16, 256, 8, 8, 300
    n_pages = (1 << 32) // (P * Hkv * D * 2) + 64
    Kp = torch.empty((n_pages, Hkv, P, D), dtype=t, device="cuda")
    Vp = torch.empty_like(Kp)
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32).cuda()
    lens = torch.tensor([n], dtype=torch.int32).cuda()
    k, v, q = values((n, Hkv, D), t, 1), values((n, Hkv, D), t, 2), values((1, Hq, D), t, 3)
    pg = ds.pages(n_pages, P, Hkv, D, 1, 2, code)
    ds.ds_append_paged(k.cuda(), v.cuda(), Kp, Vp, torch.tensor([0, n], dtype=torch.int32).cuda(), None,
                       torch.zeros(1, dtype=torch.int32).cuda(), table, pg, 1)
    out = torch.zeros((1, Hq, D), device="cuda")
    ds.ds_paged_decode(q.cuda(), Kp, Vp, out, None, lens, table, ds.ds_paged_workspace_alloc(pg, 1, Hq, n), pg, 1, Hq, n)
    prm = ds.prompt(1, Hq, Hkv, D, 1, n, code)
    out2 = torch.zeros((1, Hq, D), dtype=t, device="cuda")
    ds.ds_prompt_attention_paged(q.cuda(), Kp, Vp, out2, torch.tensor([0, 1], dtype=torch.int32).cuda(), None, lens, table,
                                 ds.ds_prompt_workspace_alloc(prm), prm, pg)
    torch.cuda.synchronize()
    near(out[0], q[0], k, v, t)
    from test_prompt import near as near_prompt
    near_prompt(out2, q, k, v, n - 1, t)


@pytest.mark.gpu
@pytest.mark.parametrize("guide", [0, 20000])
@pytest.mark.parametrize("dtype", TYPES)
def test_decode_scores_of_minus_infinity_and_nan(dtype, guide):
    """A token whose score is -infinity has no weight, wherever it lies among the wavefronts and the parts; a sequence of them alone
    is 0 / 0; a key that is NaN makes its sequence NaN, where it is the only one of its tile too."""
    t, code = TYPES[dtype]
    Hq, Hkv, P, keys = 4, 2, 32, [3000, 17, 500, 40, 65, 2000]
    Kp, Vp, table, kv = paged(keys, Hkv, P, t, 33)
    q = values((len(keys), Hq, D), t, 1)
    q[:, :, 0] = 1.0
    first = [2900, 16, 100, 40, 0, 1]        # tokens of weight 0, from the first on
    for i, n in enumerate(first):
        for j in range(n):
            Kp[table[i + 1, j // P], :, j % P, 0] = -math.inf
    Kp[table[5, 64 // P], :, 64 % P, 3] = math.nan     # the last token of the sequence of 65
    Kp[table[6, 1999 // P], :, 1999 % P, 3] = math.nan
    lens, rows = torch.tensor([7] + keys + [7], dtype=torch.int32).cuda(), torch.arange(1, len(keys) + 1, dtype=torch.int32).cuda()
    pg = ds.pages(Kp.shape[0], P, Hkv, D, table.shape[0], table.shape[1], code)
    out = torch.full((len(keys), Hq, D), CANARY, device="cuda")
    ds.ds_paged_decode(q.cuda(), Kp, Vp, out, rows, lens, table, ds.ds_paged_workspace_alloc(pg, len(keys), Hq, guide), pg, len(keys), Hq, guide)
    torch.cuda.synchronize()
    assert torch.isnan(out[3:]).all()
    for i in range(3):
        near(out[i], q[i], kv[i][0][first[i]:], kv[i][1][first[i]:], t)


@pytest.mark.gpu
@pytest.mark.parametrize("guide", [0, 20000])
@pytest.mark.parametrize("size", [1e35, 3.3895e38, 1e-20])
def test_decode_over_the_range_of_bf16(size, guide):
    """Values as large as bf16 has, in one token and in all of them, in one part and in many: the result is a number, theirs."""
    t, code, P, Hq, Hkv, keys = torch.bfloat16, ds.DS_BF16, 16, 8, 2, [1, 17, 64, 300, 3000, 20011]
    Kp, Vp, table, kv = paged(keys, Hkv, P, t, 36)
    for i, x in enumerate(kv):
        v = x[1].float()
        v = torch.where(torch.arange(D) % 3 == 0, torch.full_like(v, size), (v / v.abs().max() * size)).to(t)   # (equal ones add up)
        assert torch.isfinite(v).all()
        x[1] = v
        for j in range((keys[i] + P - 1) // P):
            part = v[j * P:(j + 1) * P].transpose(0, 1)
            Vp[table[i + 1, j], :, :part.shape[1]] = part.cuda()
    q = values((len(keys), Hq, D), t, 1)
    q[:, 0] = 0.0                                  # (equal weights)
    lens, rows = torch.tensor([7] + keys + [7], dtype=torch.int32).cuda(), torch.arange(1, len(keys) + 1, dtype=torch.int32).cuda()
    pg = ds.pages(Kp.shape[0], P, Hkv, D, table.shape[0], table.shape[1], code)
    out = torch.full((len(keys), Hq, D), CANARY, device="cuda")
    ds.ds_paged_decode(q.cuda(), Kp, Vp, out, rows, lens, table, ds.ds_paged_workspace_alloc(pg, len(keys), Hq, guide), pg, len(keys), Hq, guide)
    torch.cuda.synchronize()
    for i in range(len(keys)):
        near(out[i] / size, q[i], kv[i][0], kv[i][1].double() / size, t)


@pytest.mark.gpu
@pytest.mark.parametrize("guide", [0, 20000])
@pytest.mark.parametrize("dtype", TYPES)
def test_decode_values_that_are_not_finite(dtype, guide):
    """An infinite or NaN value is in the result of its own channel and KV head, in whichever tile and part it lies, and nowhere else."""
    t, code = TYPES[dtype]
    Hq, Hkv, P, keys = 8, 2, 32, [3000, 17, 500, 1, 65, 2000]
    Kp, Vp, table, kv = paged(keys, Hkv, P, t, 37)
    q = values((len(keys), Hq, D), t, 1)
    touched = torch.zeros((len(keys), Hq, D), dtype=torch.bool)
    for i, token, head, channel, x in ((0, 2999, 0, 5, math.inf), (0, 100, 1, 77, -math.inf), (1, 16, 1, 0, math.nan), (2, 0, 0, 127, -math.inf),
                                       (4, 64, 0, 9, math.inf), (4, 3, 0, 9, -math.inf), (5, 1024, 1, 64, math.inf)):
        Vp[table[i + 1, token // P], head, token % P, channel] = x
        touched[i, head * Hq // Hkv:(head + 1) * Hq // Hkv, channel] = True
    lens, rows = torch.tensor([7] + keys + [7], dtype=torch.int32).cuda(), torch.arange(1, len(keys) + 1, dtype=torch.int32).cuda()
    pg = ds.pages(Kp.shape[0], P, Hkv, D, table.shape[0], table.shape[1], code)
    out = torch.full((len(keys), Hq, D), CANARY, device="cuda")
    ds.ds_paged_decode(q.cuda(), Kp, Vp, out, rows, lens, table, ds.ds_paged_workspace_alloc(pg, len(keys), Hq, guide), pg, len(keys), Hq, guide)
    got = out.cpu()
    assert torch.equal(~torch.isfinite(got), touched)
    for i in range(len(keys)):      # (those channels: as if the value were a number, which the others do not depend on)
        y = defined(q[i][None], kv[i][0], kv[i][1], keys[i] - 1)[0][0].float()
        near(torch.where(touched[i], y, got[i]), q[i], kv[i][0], kv[i][1], t)


@pytest.mark.gpu
def test_decode_with_the_largest_guide():
    """max_len of 2^31 - 1 plans for long sequences, not for none: all compute units share one of 60000 tokens."""
    t, code, P, Hq, Hkv, n = torch.float16, ds.DS_F16, 64, 4, 1, 60000
    Kp, Vp, table, kv = paged([n], Hkv, P, t, 38)
    table, lens, q = table[1:2].contiguous(), torch.tensor([n], dtype=torch.int32).cuda(), values((1, Hq, D), t, 1).cuda()
    pg = ds.pages(Kp.shape[0], P, Hkv, D, 1, table.shape[1], code)
    took = []
    for guide in (n, 2**31 - 1):
        out, ws = torch.zeros((1, Hq, D), device="cuda"), ds.ds_paged_workspace_alloc(pg, 1, Hq, guide)
        run = lambda: ds.ds_paged_decode(q, Kp, Vp, out, None, lens, table, ws, pg, 1, Hq, guide)  # noqa: E731
        run()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(20):
            run()
        b.record()
        torch.cuda.synchronize()
        took.append(a.elapsed_time(b) * 50)
        near(out[0], q[0], kv[0][0], kv[0][1], t)
    print(f"{took[0]:.0f} and {took[1]:.0f} us")
    assert took[1] < 4 * took[0]


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(2, 2), (24, 2)], ids=str)
def test_decode_workspace_serves_other_batches(heads):
    """One workspace, cleared once, for more and fewer sequences in turn: what one call leaves of its parts is not where
    another counts its workgroups."""
    t, code, P, (Hq, Hkv) = torch.float16, ds.DS_F16, 32, heads
    keys = [3000, 5, 9000, 64, 65] + [100 + 7 * i for i in range(60)]
    Kp, Vp, table, kv = paged(keys, Hkv, P, t, 34)
    q = values((len(keys), Hq, D), t, 1).cuda()
    pg = ds.pages(Kp.shape[0], P, Hkv, D, table.shape[0], table.shape[1], code)
    ws = ds.ds_paged_workspace_alloc(pg, len(keys), Hq, 0)
    lens, rows = torch.tensor([7] + keys + [7], dtype=torch.int32).cuda(), torch.arange(1, len(keys) + 1, dtype=torch.int32).cuda()
    for n, guide in ((1, 3000), (65, 9000), (3, 9000), (65, 0), (2, 100000), (30, 9000), (65, 9000)):
        out = torch.full((n, Hq, D), CANARY, device="cuda")
        ds.ds_paged_decode(q[:n], Kp, Vp, out, rows[:n], lens, table, ws, pg, n, Hq, guide)
        torch.cuda.synchronize()
        for i in range(n):
            near(out[i], q[i], kv[i][0], kv[i][1], t)


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(8, 8), (32, 2)], ids=str)
@pytest.mark.parametrize("n", [1, 4, 40])
def test_decode_short_beside_long(n, heads):
    """Units that are not cut (up to 256 tokens) between units that are, wherever the shares' ends fall; the guide, and with it
    the number of shares, from one to all that there are."""
    t, code, P, (Hq, Hkv) = torch.bfloat16, ds.DS_BF16, 16, heads
    keys = ([5, 3000, 257, 256, 20, 5000, 64, 320, 321, 1, 700, 0, 255, 1500] * 3)[:n]
    Kp, Vp, table, kv = paged(keys, Hkv, P, t, 35)
    q = values((n, Hq, D), t, 1).cuda()
    lens, rows = torch.tensor([7] + keys + [7], dtype=torch.int32).cuda(), torch.arange(1, n + 1, dtype=torch.int32).cuda()
    pg = ds.pages(Kp.shape[0], P, Hkv, D, table.shape[0], table.shape[1], code)
    ws = ds.ds_paged_workspace_alloc(pg, n, Hq, 0)
    for guide in (0, 64, 200, 1000, 100000):
        out = torch.full((n, Hq, D), CANARY, device="cuda")
        ds.ds_paged_decode(q, Kp, Vp, out, rows, lens, table, ws, pg, n, Hq, guide)
        torch.cuda.synchronize()
        for i in range(n):
            if keys[i]:
                near(out[i], q[i], kv[i][0], kv[i][1], t)
            else:
                assert (out[i] == 0).all()


# ------------------------------------------------------------------ append
@pytest.mark.gpu
@pytest.mark.parametrize("Hkv", [1, 3, 8, 40])
@pytest.mark.parametrize("P", [16, 64])
def test_append(P, Hkv):
    """Rows land where the table says, everything else of the pools stays; sequences without a place are passed over."""
    t = torch.bfloat16
    new, begin = [1, 0, 37, 5, 4, 2, 130], [15, 3, 0, 60, -1, 2 * 16 * 40, 7]
    n, first, pages = len(new), 3, 40
    T = sum(new) + first + 2
    wide = values((T, 2 * Hkv + 1, D), t, 1).cuda()
    k, v = wide[:, :Hkv], wide[:, Hkv:2 * Hkv]
    order = torch.randperm(n * 12, generator=torch.Generator().manual_seed(2)).to(torch.int32).reshape(n, 12)
    order[3, 4 if P == 16 else 1] = n * 12           # (that page is not one of the pool)
    table = torch.full((n + 1, 12), -1, dtype=torch.int32)
    rows = torch.tensor([2, 0, 1, 3, 4, 5, 7], dtype=torch.int32)
    table = torch.full((8, 12), -1, dtype=torch.int32)
    table[rows.long()] = order
    new_start = torch.tensor([first] + [first + sum(new[:i + 1]) for i in range(n)], dtype=torch.int32)
    pools = torch.randn((2, n * 12, Hkv, P, D), generator=torch.Generator().manual_seed(3)).to(t)
    want = pools.clone()
    for s in range(n):
        for i in range(new[s]):
            at = begin[s] + i
            if begin[s] < 0 or at // P >= 12 or not 0 <= order[s, at // P] < n * 12:
                continue
            want[0, order[s, at // P], :, at % P] = k[new_start[s] + i].cpu()
            want[1, order[s, at // P], :, at % P] = v[new_start[s] + i].cpu()
    K, V = pools[0].contiguous().cuda(), pools[1].contiguous().cuda()
    pg = ds.pages(n * 12, P, Hkv, D, 8, 12, ds.DS_BF16)
    ds.ds_append_paged(k, v, K, V, new_start.cuda(), rows.cuda(), torch.tensor(begin, dtype=torch.int32).cuda(), table.cuda(), pg, n)
    torch.cuda.synchronize()
    assert torch.equal(K.cpu().view(torch.int16), want[0].view(torch.int16)) and torch.equal(V.cpu().view(torch.int16), want[1].view(torch.int16))


@pytest.mark.gpu
@pytest.mark.parametrize("Hkv", [1, 2])
def test_append_rows_of_any_dense_view(Hkv):
    """One token or one head by transposition: that dimension's stride says nothing."""
    P, t = 16, torch.float16
    pg = ds.pages(3, P, Hkv, D, 1, 3)
    table, new_start = torch.tensor([[2, 0, 1]], dtype=torch.int32).cuda(), lambda n: torch.tensor([0, n], dtype=torch.int32).cuda()
    for n in (1, 5):
        for form in ("dense", "heads_first", "slice"):
            if form == "slice":
                k, v = (values((n, Hkv + 3, D), t, i).cuda()[:, 1:1 + Hkv] for i in (1, 2))
            elif form == "dense":
                k, v = (values((n, Hkv, D), t, i).cuda() for i in (1, 2))
            elif n == 1 or Hkv == 1:
                k, v = (values((Hkv, n, D), t, i).cuda().transpose(0, 1) for i in (1, 2))
            else:
                continue
            K = torch.zeros((3, Hkv, P, D), dtype=t, device="cuda")
            V = torch.zeros_like(K)
            ds.ds_append_paged(k, v, K, V, new_start(n), None, torch.tensor([18], dtype=torch.int32).cuda(), table, pg, 1)
            want = torch.zeros_like(K), torch.zeros_like(K)
            for w, x in zip(want, (k, v)):
                w[0, :, 2:2 + n] = x.transpose(0, 1)
            assert torch.equal(K, want[0]) and torch.equal(V, want[1]), (n, form)


def test_append_rows_that_cannot_be():
    pg = ds.pages(**PG)
    x, i = torch.zeros(4, 2, D), torch.zeros(4, dtype=torch.int32)
    for k, v in ((x[:, :1], x[:, :1]), (x[..., :64], x[..., :64]), (x[:3], x), (x, x[::2].repeat(2, 1, 1)[:3]), (x.transpose(0, 1).contiguous().transpose(0, 1), x),
                 (torch.zeros(4, D, 2).transpose(1, 2), x), (torch.zeros(4, 3, D)[:, :2], x)):
        with pytest.raises(ValueError, match="new rows|the same"):
            ds.ds_append_paged(k, v, x, x, i, i, i, i, pg, 1)
