"""The books of a paged cache: refusals on the host; extend, fork, free, compact and copy against a model that
does the same one page at a time; and a serving run of all of it, with prompts and decode, eager, on two streams
and captured."""
import ctypes

import pytest
import torch

import paper_2408_07092_amd as ds
from test_paged import BAD_PAGES, OFF, PG, near
from test_prompt import D, FAKE, values
from test_prompt import near as near_prompt


# ------------------------------------------------------------------ host
def calls(pg, n=2):
    """Entry points with their pointers, by name: (function of the pointers, names, alignments)."""
    L, g = ds.lib(), ctypes.byref(pg) if pg else None
    return {
        "extend": (lambda p: L.ds_pages_extend(*p, g, n, None), dict(refs=16, table=4, lens=4, rows=4, n_new=4, start=4, status=4)),
        "fork": (lambda p: L.ds_pages_fork(*p, g, n, None), dict(refs=16, table=4, lens=4, src=4, dst=4, copies=16, n_copies=4, status=4)),
        "free": (lambda p: L.ds_pages_free(*p, g, n, None), dict(refs=16, table=4, lens=4, rows=4, status=4)),
        "compact": (lambda p: L.ds_pages_compact(*p, 1 << 30, g, None), dict(refs=16, table=4, lens=4, copies=16, n_copies=4, status=4, ws=16)),
        "copy": (lambda p: L.ds_pages_copy(*p, g, n, None), dict(K=256, V=256, copies=16, n_copies=4)),
    }


def test_refusals():
    for name, (f, args) in calls(ds.pages(**PG)).items():
        for i, by in enumerate(args.values()):
            p = [FAKE] * len(args)
            p[i] = None
            assert f(p) == ds.DS_ERR_NULL, (name, i)
            p[i] = OFF[by]
            assert f(p) == ds.DS_ERR_ALIGN, (name, i)
        assert calls(None)[name][0]([FAKE] * len(args)) == ds.DS_ERR_NULL
        for bad in BAD_PAGES:
            assert calls(ds.pages(**{**PG, **bad}))[name][0]([FAKE] * len(args)) == ds.DS_ERR_SHAPE, (name, bad)
        if name in ("extend", "fork", "free"):
            for n in (0, -1, 2049):
                assert calls(ds.pages(**PG), n)[name][0]([FAKE] * len(args)) == ds.DS_ERR_SHAPE, (name, n)
    copy = lambda n, **more: calls(ds.pages(**{**PG, **more}), n)["copy"][0]([FAKE] * 4)  # noqa: E731
    assert copy(-1) == ds.DS_ERR_SHAPE and copy(2**31 - 1) == ds.DS_ERR_SHAPE and copy(0) == ds.DS_OK
    assert ds.ds_pages_workspace_bytes(ds.pages(**PG)) >= 80 and ds.lib().ds_pages_workspace_bytes(None) == 0
    assert ds.lib().ds_pages_compact(*[FAKE] * 7, 79, ctypes.byref(ds.pages(**PG)), None) == ds.DS_ERR_WORKSPACE


# ------------------------------------------------------------------ model
class Books:
    """Counts, table and lengths, a page at a time."""

    def __init__(self, n_pages, P, n_rows, max_pages):
        self.P, self.max_pages = P, max_pages
        self.refs, self.lens = [0] * n_pages, [0] * n_rows
        self.table = [[-1] * max_pages for _ in range(n_rows)]

    def pages_of(self, n):
        return (n + self.P - 1) // self.P

    def lowest(self, n):
        free = [p for p, r in enumerate(self.refs) if r == 0]
        return free[:n] if len(free) >= n else None

    def bad_rows(self, rows):
        return len(set(rows)) < len(rows) or any(not 0 <= r < len(self.lens) for r in rows)

    def extend(self, rows, n_new):
        if self.bad_rows(rows):
            return ds.DS_PAGES_ROWS, [-1] * len(rows)
        if any(n < 0 or self.lens[r] + n > self.max_pages * self.P for r, n in zip(rows, n_new)):
            return ds.DS_PAGES_LENGTH, [-1] * len(rows)
        need = [self.pages_of(self.lens[r] + n) - self.pages_of(self.lens[r]) for r, n in zip(rows, n_new)]
        got = self.lowest(sum(need))
        if got is None:
            return ds.DS_PAGES_NO_ROOM, [-1] * len(rows)
        start = []
        for r, n, k in zip(rows, n_new, need):
            at = self.pages_of(self.lens[r])
            for j in range(k):
                p = got.pop(0)
                self.table[r][at + j], self.refs[p] = p, 1
            start.append(self.lens[r])
            self.lens[r] += n
        return ds.DS_PAGES_DONE, start

    def fork(self, src, dst):
        if (self.bad_rows(dst) or any(not 0 <= r < len(self.lens) for r in src) or set(src) & set(dst) or any(self.lens[r] for r in dst)):
            return ds.DS_PAGES_ROWS, []
        half = [self.lens[r] % self.P for r in src]
        got = self.lowest(sum(h > 0 for h in half))
        if got is None:
            return ds.DS_PAGES_NO_ROOM, []
        copies = []
        for s, d, h in zip(src, dst, half):
            full = self.lens[s] // self.P
            for j in range(full):
                self.table[d][j] = self.table[s][j]
                self.refs[self.table[s][j]] += 1
            if h:
                p = got.pop(0)
                copies.append([self.table[s][full], p, h, 0])
                self.table[d][full], self.refs[p] = p, 1
            self.lens[d] = self.lens[s]
        return ds.DS_PAGES_DONE, copies

    def free(self, rows):
        if self.bad_rows(rows):
            return ds.DS_PAGES_ROWS
        for r in rows:
            for j in range(self.pages_of(self.lens[r])):
                self.refs[self.table[r][j]] -= 1
                self.table[r][j] = -1
            self.lens[r] = 0
        return ds.DS_PAGES_DONE

    def compact(self):
        live = [p for p, r in enumerate(self.refs) if r > 0]
        movers = [p for p in live if p >= len(live)]
        holes = [p for p in range(len(live)) if self.refs[p] == 0]
        to = dict(zip(movers, holes))
        for p, h in to.items():
            self.refs[h], self.refs[p] = self.refs[p], 0
        for r, n in enumerate(self.lens):
            for j in range(self.pages_of(n)):
                self.table[r][j] = to.get(self.table[r][j], self.table[r][j])
        return [[p, h, self.P, 0] for p, h in to.items()]


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Device:
    """The same through the library."""

    def __init__(self, n_pages, P, n_rows, max_pages, Hkv=1):
        self.pg = ds.pages(n_pages, P, Hkv, D, n_rows, max_pages)
        self.refs, self.lens = ints([0] * n_pages), ints([0] * n_rows)
        self.table = torch.full((n_rows, max_pages), -1, dtype=torch.int32, device="cuda")
        self.ws = ds.ds_pages_workspace_alloc(self.pg)

    def extend(self, rows, n_new):
        start, status = ints([77] * (len(rows) + 1)), ints([77])
        ds.ds_pages_extend(self.refs, self.table, self.lens, ints(rows), ints(n_new), start, status, self.pg, len(rows))
        assert start[-1].item() == 77
        return status.item(), start[:-1].tolist()

    def fork(self, src, dst):
        copies, count, status = ints([[77] * 4] * (len(src) + 1)), ints([77]), ints([77])
        ds.ds_pages_fork(self.refs, self.table, self.lens, ints(src), ints(dst), copies, count, status, self.pg, len(src))
        n = count.item()
        assert 0 <= n <= len(src) and (copies[n:] == 77).all()
        return status.item(), copies[:n].tolist()

    def free(self, rows):
        status = ints([77])
        ds.ds_pages_free(self.refs, self.table, self.lens, ints(rows), status, self.pg, len(rows))
        return status.item()

    def compact(self):
        copies, count, status = ints([[77] * 4] * (self.pg.n_pages // 2 + 1)), ints([77]), ints([77])
        ds.ds_pages_compact(self.refs, self.table, self.lens, copies, count, status, self.ws, self.pg)
        n = count.item()
        assert status.item() == ds.DS_PAGES_DONE and (copies[n:] == 77).all()
        return copies[:n].tolist()

    def same(self, b):
        assert self.refs.tolist() == b.refs and self.lens.tolist() == b.lens and self.table.tolist() == b.table


def test_tensors_off_the_device_are_refused():
    """Memory of the host, which a kernel could not read, does not get as far as a launch."""
    x, i, pg, prm = torch.zeros(1, 1, D), torch.zeros(4, dtype=torch.int32), ds.pages(1, 16, 1, D, 1, 1), ds.prompt(1, 1, 1, D, 1, 1)
    for call in (lambda: ds.ds_prompt_attention(x, x, x, x, i, i, i, x, prm), lambda: ds.ds_prompt_attention_paged(x, x, x, x, i, i, i, i, x, prm, pg),
                 lambda: ds.ds_paged_decode(x, x, x, x, i, i, i, x, pg, 1, 1, 1), lambda: ds.ds_append_paged(x, x, x, x, i, i, i, i, pg, 1),
                 lambda: ds.ds_pages_extend(i, i, i, i, i, i, i, pg, 1), lambda: ds.ds_pages_fork(i, i, i, i, i, i, i, i, pg, 1),
                 lambda: ds.ds_pages_free(i, i, i, i, i, pg, 1), lambda: ds.ds_pages_compact(i, i, i, i, i, i, x, pg),
                 lambda: ds.ds_pages_copy(x, x, i, i, pg, 1)):
        with pytest.raises(ValueError, match="not the current device"):
            call()


class Placed:
    """What a call asks of a tensor before a launch: where it is and what shape it has."""
    def __init__(self, device, shape=(4, 1, D), dtype=2):
        self.at, self.shape, self.dtype, self.device = device, shape, dtype, f"place {device}"

    def get_device(self):
        return self.at

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x10000

    def stride(self, i=None):
        return (D, D, 1) if i is None else (D, D, 1)[i]

    def numel(self):
        return 1 << 20

    def element_size(self):
        return self.dtype


@pytest.mark.parametrize("where", [-1, 1])      # (the host; another device)
def test_every_tensor_of_a_call_is_looked_at(monkeypatch, where):
    """One tensor that is not on the current device, in each place of each call: refused ahead of the library, and so is a stream
    of another device."""
    reached = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: reached.append(name) or 0
    monkeypatch.setattr(ds.binding, "lib", lambda: Library())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    pg, prm = ds.pages(1, 16, 1, D, 1, 1), ds.prompt(1, 1, 1, D, 1, 1)
    stream = type("Stream", (), {"device_index": 1, "device": "place 1", "cuda_stream": 0})()
    for f, n, more in ((ds.ds_prompt_attention, 8, (prm,)), (ds.ds_prompt_attention_paged, 9, (prm, pg)), (ds.ds_paged_decode, 8, (pg, 1, 1, 1)),
                       (ds.ds_append_paged, 8, (pg, 1)), (ds.ds_pages_extend, 7, (pg, 1)), (ds.ds_pages_fork, 8, (pg, 1)),
                       (ds.ds_pages_free, 5, (pg, 1)), (ds.ds_pages_compact, 7, (pg,)), (ds.ds_pages_copy, 4, (pg, 1))):
        f(*[Placed(0)] * n, *more)
        assert reached.pop() == f.__name__
        for i in range(n):
            with pytest.raises(ValueError, match="not the current device"):
                f(*[Placed(where if j == i else 0) for j in range(n)], *more)
        with pytest.raises(ValueError, match="not the current device"):
            f(*[Placed(0)] * n, *more, stream=stream)
        assert not reached, f.__name__


def test_workspaces_are_memory_of_a_gpu():
    for alloc in (lambda: ds.ds_prompt_workspace_alloc(ds.prompt(1, 1, 1, D, 1, 1), "cpu"), lambda: ds.ds_paged_workspace_alloc(ds.pages(1, 16, 1, D, 1, 1), 1, 1, 1, "cpu"),
                  lambda: ds.ds_pages_workspace_alloc(ds.pages(1, 16, 1, D, 1, 1), "cpu")):
        with pytest.raises(ValueError, match="memory of a GPU"):
            alloc()


@pytest.mark.gpu
@pytest.mark.parametrize("n_pages,P,n_rows,max_pages", [(1, 16, 3, 2), (40, 16, 12, 7), (900, 32, 30, 60), (17000, 16, 70, 700), (40000, 256, 40, 1500)])
def test_books_against_the_model(n_pages, P, n_rows, max_pages):
    """Long runs of calls, refused ones among them: after each the books are the model's, to the last entry."""
    rng = torch.Generator().manual_seed(n_pages)
    pick = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=rng))  # noqa: E731
    dev, mod = Device(n_pages, P, n_rows, max_pages), Books(n_pages, P, n_rows, max_pages)
    seen = set()
    for step in range(60):
        some = torch.randperm(n_rows, generator=rng).tolist()[:pick(1, n_rows)]
        kind = ("extend", "extend", "fork", "free", "compact")[pick(0, 4)] if step else "extend"
        if kind == "extend":
            top = (1, P, 3 * P, max_pages * P // 2)[pick(0, 3)]
            args = (some, [pick(0, top) for _ in some])
        elif kind == "fork":
            empty = [r for r in range(n_rows) if mod.lens[r] == 0] or some[:1]
            full = [r for r in range(n_rows) if mod.lens[r] > 0] or some[:1]
            args = ([full[pick(0, len(full) - 1)] for _ in empty], empty)
        else:
            args = (some[:max(1, len(some) // 2)],) if kind == "free" else ()
        if kind != "compact" and pick(0, 5) == 0:       # a list that is wrong
            rows = args[-1] if kind == "fork" else args[0]
            at = pick(0, len(rows) - 1)
            rows[at] = (-1, n_rows, rows[0] if at else 2**31 - 1)[pick(0, 2)]
        got, want = getattr(dev, kind)(*args), getattr(mod, kind)(*args)
        assert got == want, (step, kind, args)
        dev.same(mod)
        seen.add((kind, want if kind == "free" else want[0] if kind != "compact" else bool(want)))
    assert len(seen) >= 4


@pytest.mark.gpu
def test_books_at_their_limits():
    """Lists of 2048 rows, more pages at a time than are remembered, the last page of 2^20, and none left."""
    dev, mod = Device(6000, 16, 2100, 3000), Books(6000, 16, 2100, 3000)
    rows = list(range(2048))[::-1]
    assert dev.extend(rows, [17] * 2048) == mod.extend(rows, [17] * 2048)
    assert dev.extend([2050], [16 * 1904]) == mod.extend([2050], [16 * 1904])       # the last free page
    dev.same(mod)
    assert dev.extend([2051], [1]) == (ds.DS_PAGES_NO_ROOM, [-1]) and dev.extend([2051], [0]) == (ds.DS_PAGES_DONE, [0])
    assert dev.free(rows) == mod.free(rows)
    src, dst = [2050] * 40, list(range(40))
    assert dev.fork(src, dst) == mod.fork(src, dst)                                   # (two launches: 40 * 3000 entries)
    assert dev.compact() == mod.compact()
    dev.same(mod)
    big = Device(1 << 20, 16, 2, 1 << 20)
    assert big.extend([0, 1], [16 * (1 << 19)] * 2) == (ds.DS_PAGES_DONE, [0, 0])
    want = torch.arange(1 << 20, dtype=torch.int32, device="cuda").reshape(2, 1 << 19)
    assert torch.equal(big.table[:, :1 << 19], want) and (big.table[:, 1 << 19:] == -1).all() and (big.refs == 1).all()
    assert big.free([0]) == ds.DS_PAGES_DONE
    assert len(big.compact()) == 1 << 19 and (big.refs[:1 << 19] == 1).all() and (big.refs[1 << 19:] == 0).all()
    assert torch.equal(big.table[1, :1 << 19], want[0])
    assert big.extend([1], [16 * (1 << 19)]) == (ds.DS_PAGES_DONE, [16 * (1 << 19)])
    assert big.extend([0], [1])[0] == ds.DS_PAGES_NO_ROOM and big.extend([1], [2**31 - 1])[0] == ds.DS_PAGES_LENGTH


@pytest.mark.gpu
@pytest.mark.parametrize("length", [-1, -(2**31), 7 * 16 + 1, 2**31 - 1])
def test_free_reports_a_length_that_cannot_be(length):
    """... and changes nothing, in whichever place of the list the row is; a row that is none counts for more."""
    dev, mod = Device(40, 16, 12, 7), Books(40, 16, 12, 7)
    rows, n = [3, 0, 11, 5], [40, 112, 1, 17]
    assert dev.extend(rows, n) == mod.extend(rows, n)
    dev.lens[5] = mod.lens[5] = length
    for wrong in ([5], [3, 5], [5, 11, 0], [0, 3, 5, 11]):
        assert dev.free(wrong) == ds.DS_PAGES_LENGTH
        dev.same(mod)
    assert dev.free([5, 12]) == ds.DS_PAGES_ROWS and dev.free([5, 3, 5]) == ds.DS_PAGES_ROWS
    dev.same(mod)
    assert dev.free([11, 3]) == mod.free([11, 3]) == ds.DS_PAGES_DONE
    dev.same(mod)


@pytest.mark.gpu
@pytest.mark.parametrize("length", [-1, 7 * 16 + 1, 2**31 - 1])
@pytest.mark.parametrize("row", [0, 1999])
def test_compact_reports_a_length_that_cannot_be(row, length):
    dev, mod = Device(2000, 16, 2000, 7), Books(2000, 16, 2000, 7)
    rows = [row, 5, 700]
    assert dev.extend(rows, [40, 112, 17]) == mod.extend(rows, [40, 112, 17])
    assert dev.free([5]) == mod.free([5]) and dev.extend([3], [20]) == mod.extend([3], [20])
    dev.lens[row] = mod.lens[row] = length
    copies, count, status = ints([[77] * 4] * 1001), ints([77]), ints([77])
    ds.ds_pages_compact(dev.refs, dev.table, dev.lens, copies, count, status, dev.ws, dev.pg)
    assert status.item() == ds.DS_PAGES_LENGTH and count.item() == 0 and (copies == 77).all()
    dev.same(mod)
    dev.lens[row] = mod.lens[row] = 40
    assert dev.compact() == mod.compact()
    dev.same(mod)


@pytest.mark.gpu
@pytest.mark.parametrize("n_pages", [50, 16384 + 50])
def test_compact_leaves_entries_of_pages_that_nobody_holds(n_pages):
    """... which books in order do not have: what the workspace held before does not get into the table."""
    dev, mod = Device(n_pages, 16, 4, 30), Books(n_pages, 16, 4, 30)
    for r, p in ((0, n_pages - 1), (0, n_pages - 2), (1, 7), (1, n_pages - 5), (2, 1)):
        at = mod.lens[r] // 16
        mod.table[r][at] = dev.table[r, at] = p
        mod.lens[r] += 16
        if p != n_pages - 2:
            mod.refs[p] = 1
    dev.refs, dev.lens = ints(mod.refs), ints(mod.lens)
    dev.ws.fill_(0x11)
    assert dev.compact() == mod.compact()
    dev.same(mod)
    assert dev.table[0, 1].item() == n_pages - 2


@pytest.mark.gpu
@pytest.mark.parametrize("Hkv", [1, 3, 8])
@pytest.mark.parametrize("P", [16, 64, 256])
def test_copy(P, Hkv):
    n_pages = 50
    pools = torch.randn((2, n_pages, Hkv, P, D), generator=torch.Generator().manual_seed(1)).half().cuda()
    copies = [[3, 40, P, 0], [4, 41, 1, 0], [3, 42, P - 1, 0], [5, 43, 0, 0], [n_pages, 44, P, 0], [6, -1, P, 0], [7, n_pages, P, 0],
              [8, 45, P + 9, 0], [9, 46, -2, 0], [10, 47, 9, 0], [11, 48, P, 0]]
    want = pools.clone()
    for src, dst, n, _ in copies[:10]:
        if 0 <= src < n_pages and 0 <= dst < n_pages and n > 0:
            want[:, dst, :, :n] = want[:, src, :, :n]
    pg = ds.pages(n_pages, P, Hkv, D, 1, 1)
    ds.ds_pages_copy(pools[0], pools[1], ints(copies), ints([10]), pg, 11)
    assert torch.equal(pools, want)
    ds.ds_pages_copy(pools[0], pools[1], ints(copies), ints([-4]), pg, 11)
    assert torch.equal(pools, want)
    want[:, 48] = want[:, 11]
    ds.ds_pages_copy(pools[0], pools[1], ints(copies), ints([99]), pg, 11)
    assert torch.equal(pools, want)


# ------------------------------------------------------------------ together
class Server:
    """Sequences over one layer's pages as a program runs them, and beside them every sequence's rows by themselves."""

    def __init__(self, t, code, P=16, Hq=8, Hkv=2, n_pages=120, n_rows=8, max_pages=40):
        self.t, self.Hq, self.Hkv = t, Hq, Hkv
        self.dev = Device(n_pages, P, n_rows, max_pages, Hkv)
        self.dev.pg = ds.pages(n_pages, P, Hkv, D, n_rows, max_pages, code)
        self.K = torch.full((n_pages, Hkv, P, D), float("nan"), dtype=t, device="cuda")
        self.V = self.K.clone()
        self.rows = {}
        self.seed, self.code = 0, code

    def take_in(self, new):
        """Prompts, or parts of them: {row: tokens}."""
        d, ids, n = self.dev, list(new), list(new.values())
        self.seed += 1
        T = sum(n)
        fused = values((T, self.Hq + 2 * self.Hkv, D), self.t, self.seed).cuda()
        q, k, v = fused[:, :self.Hq], fused[:, self.Hq:self.Hq + self.Hkv], fused[:, self.Hq + self.Hkv:]
        starts = ints([sum(n[:i]) for i in range(len(n) + 1)])
        start, status, rows = ints([0] * len(n)), ints([9]), ints(ids)
        ds.ds_pages_extend(d.refs, d.table, d.lens, rows, ints(n), start, status, d.pg, len(n))
        ds.ds_append_paged(k, v, self.K, self.V, starts, rows, start, d.table, d.pg, len(n))
        prm = ds.prompt(len(n), self.Hq, self.Hkv, D, T, 600, self.code, q_stride=fused.stride(0))
        out = torch.zeros((T, self.Hq, D), dtype=self.t, device="cuda")
        ds.ds_prompt_attention_paged(q, self.K, self.V, out, starts, rows, d.lens, d.table, ds.ds_prompt_workspace_alloc(prm), prm, d.pg)
        assert status.item() == 0
        at = 0
        for r, m in new.items():
            old = self.rows.get(r)
            kv = torch.stack((k[at:at + m], v[at:at + m]))
            self.rows[r] = kv if old is None else torch.cat((old, kv), 1)
            before = self.rows[r].shape[1] - m
            near_prompt(out[at:at + m], q[at:at + m], self.rows[r][0], self.rows[r][1], before, self.t)
            at += m

    def branch(self, src, dst):
        d = self.dev
        copies, count, status = ints([[0] * 4] * len(src)), ints([0]), ints([9])
        ds.ds_pages_fork(d.refs, d.table, d.lens, ints(src), ints(dst), copies, count, status, d.pg, len(src))
        ds.ds_pages_copy(self.K, self.V, copies, count, d.pg, len(src))
        assert status.item() == 0
        for s, t in zip(src, dst):
            self.rows[t] = self.rows[s]

    def end(self, ids):
        assert self.dev.free(ids) == 0
        for r in ids:
            del self.rows[r]

    def close_up(self):
        d = self.dev
        copies, count, status = ints([[0] * 4] * (d.pg.n_pages // 2 + 1)), ints([0]), ints([9])
        ds.ds_pages_compact(d.refs, d.table, d.lens, copies, count, status, d.ws, d.pg)
        ds.ds_pages_copy(self.K, self.V, copies, count, d.pg, copies.shape[0])
        live = int((d.refs > 0).sum())
        assert status.item() == 0 and (d.refs[live:] == 0).all()

    def step_buffers(self, ids):
        n = len(ids)
        b = dict(rows=ints(ids), one=ints([1] * n), starts=ints(list(range(n + 1))), start=ints([0] * n), status=ints([9]),
                 q=torch.zeros((n, self.Hq, D), dtype=self.t, device="cuda"),
                 kv=torch.zeros((2, n, self.Hkv, D), dtype=self.t, device="cuda"),
                 out=torch.zeros((n, self.Hq, D), device="cuda"), ws=ds.ds_paged_workspace_alloc(self.dev.pg, n, self.Hq, 600))
        return b

    def enqueue(self, b, ids):
        d, n = self.dev, len(ids)
        ds.ds_pages_extend(d.refs, d.table, d.lens, b["rows"], b["one"], b["start"], b["status"], d.pg, n)
        ds.ds_append_paged(b["kv"][0], b["kv"][1], self.K, self.V, b["starts"], b["rows"], b["start"], d.table, d.pg, n)
        ds.ds_paged_decode(b["q"], self.K, self.V, b["out"], b["rows"], d.lens, d.table, b["ws"], d.pg, n, self.Hq, 600)

    def new_tokens(self, b, ids):
        self.seed += 1
        b["q"].copy_(values(b["q"].shape, self.t, self.seed))
        b["kv"].copy_(values(b["kv"].shape, self.t, self.seed + 1000))
        for i, r in enumerate(ids):
            self.rows[r] = torch.cat((self.rows[r], b["kv"][:, i:i + 1]), 1)

    def check(self, b, ids):
        assert b["status"].item() == 0
        for i, r in enumerate(ids):
            near(b["out"][i], b["q"][i], self.rows[r][0], self.rows[r][1], self.t)

    def step(self, ids):
        b = self.step_buffers(ids)
        self.new_tokens(b, ids)
        self.enqueue(b, ids)
        self.check(b, ids)


@pytest.mark.gpu
@pytest.mark.parametrize("t,code,P", [(torch.float16, ds.DS_F16, 16), (torch.bfloat16, ds.DS_BF16, 64)], ids=str)
def test_serving_run(t, code, P):
    """Prompts by parts, decode, branches that part, sequences that end, a pool closed up under way, rows used again."""
    s = Server(t, code, P)
    s.take_in({3: 33, 0: 1, 5: 100})
    s.step([0, 3, 5])
    s.take_in({5: 60, 1: 16})
    s.branch([5, 5, 1, 0], [2, 4, 6, 7])
    for _ in range(3):
        s.step([5, 4, 2, 1, 6, 7, 0])       # branches and their parents part
    s.end([5, 0, 1])
    s.close_up()
    s.step([2, 3, 4, 6, 7])
    s.take_in({0: 70, 4: 5})
    s.branch([4], [5])
    s.step([5, 0, 4, 2])
    s.end([0, 2, 3, 4, 5, 6, 7])
    assert (s.dev.refs == 0).all() and (s.dev.lens == 0).all()


@pytest.mark.gpu
def test_captured_step():
    """One captured step of extend, append and decode, replayed while the sequences grow over pages' ends; eager
    calls and new inputs between the replays."""
    s = Server(torch.float16, ds.DS_F16)
    ids = [1, 4, 6]
    s.take_in({1: 14, 4: 47, 6: 200})
    s.take_in({2: 20})
    s.step(ids)
    b = s.step_buffers(ids)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            s.enqueue(b, ids)
    for i in range(20):
        s.new_tokens(b, ids)
        graph.replay()
        s.check(b, ids)
        if i % 5 == 2:
            s.step([2])
        if i == 9:
            s.branch([2], [0])
            s.close_up()
            s.end([0])


@pytest.mark.gpu
def test_streams_and_repeats():
    """Calls with workspaces of their own on two streams at once, and the same call again and again: the same bits."""
    t, code, P, Hq, Hkv, keys = torch.bfloat16, ds.DS_BF16, 32, 16, 4, [3000, 1, 0, 700, 5001]
    from test_prompt import paged, starts
    Kp, Vp, table, _ = paged(keys, Hkv, P, t, 40)
    table, lens = table[1:-1].contiguous(), ints(keys)
    pg = ds.pages(Kp.shape[0], P, Hkv, D, len(keys), table.shape[1], code)
    q = values((len(keys), Hq, D), t, 1).cuda()
    new = [40, 1, 0, 300, 7]
    qp = values((sum(new), Hq, D), t, 2).cuda()
    prm = ds.prompt(len(keys), Hq, Hkv, D, sum(new), max(keys), code)
    work = [(torch.cuda.Stream(), ds.ds_paged_workspace_alloc(pg, len(keys), Hq, max(keys)), ds.ds_prompt_workspace_alloc(prm)) for _ in range(2)]
    qs = starts(new).cuda()
    outs = []
    torch.cuda.synchronize()
    for _ in range(8):
        for st, ws, wp in work:
            o, p = torch.empty((len(keys), Hq, D), device="cuda"), torch.empty_like(qp)
            st.wait_stream(torch.cuda.current_stream())
            ds.ds_paged_decode(q, Kp, Vp, o, None, lens, table, ws, pg, len(keys), Hq, max(keys), stream=st)
            ds.ds_prompt_attention_paged(qp, Kp, Vp, p, qs, None, lens, table, wp, prm, pg, stream=st)
            outs.append((o, p))
    torch.cuda.synchronize()
    for o, p in outs[1:]:
        assert torch.equal(o, outs[0][0]) and torch.equal(p.view(torch.int16), outs[0][1].view(torch.int16))


@pytest.mark.gpu
def test_two_captured_calls_share_a_workspace():
    """Decode and split prompts of two batches, captured apart with one workspace each for both, replayed in turn with eager calls of
    a third batch between: every time the bits of the eager calls."""
    t, code, P, Hq, Hkv, keys = torch.float16, ds.DS_F16, 16, 8, 2, [3000, 40, 0, 700, 5001]
    from test_prompt import paged, starts
    Kp, Vp, table, _ = paged(keys, Hkv, P, t, 41)
    table, lens = table[1:-1].contiguous(), ints(keys)
    pg = ds.pages(Kp.shape[0], P, Hkv, D, len(keys), table.shape[1], code)
    calls = []
    for rows, new in (([4, 0, 3], [1, 9, 30]), ([0, 1, 2, 3, 4], [5, 2, 0, 1, 16]), ([1, 4], [20, 3])):
        n, T = len(rows), sum(new)
        calls.append(dict(n=n, rows=ints(rows), q=values((n, Hq, D), t, n).cuda(), qp=values((T, Hq, D), t, 10 + n).cuda(), qs=starts(new).cuda(),
                          prm=ds.prompt(n, Hq, Hkv, D, T, 5001, code), o=torch.zeros((n, Hq, D), device="cuda"),
                          p=torch.zeros((T, Hq, D), dtype=t, device="cuda")))
    ws = ds.ds_paged_workspace_alloc(pg, 5, Hq, 5001)
    wp = torch.empty(max(ds.ds_prompt_workspace_bytes(c["prm"]) for c in calls), dtype=torch.uint8, device="cuda")
    assert wp.numel() > 256

    def run(c):
        ds.ds_paged_decode(c["q"], Kp, Vp, c["o"], c["rows"], lens, table, ws, pg, c["n"], Hq, 5001)
        ds.ds_prompt_attention_paged(c["qp"], Kp, Vp, c["p"], c["qs"], c["rows"], lens, table, wp, c["prm"], pg)

    for c in calls:
        run(c)
    torch.cuda.synchronize()
    want = [(c["o"].clone(), c["p"].clone()) for c in calls]
    graphs = []
    for c in calls[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(c)
        graphs.append(g)
    for i in range(6):
        for j in ((0, 2, 1) if i % 2 else (1, 0, 2)):
            c = calls[j]
            c["o"].fill_(7.0)
            c["p"].fill_(7.0)
            graphs[j].replay() if j < 2 else run(c)
            torch.cuda.synchronize()
            assert torch.equal(c["o"], want[j][0]) and torch.equal(c["p"], want[j][1]), (i, j)
