"""Forking, growing, freeing and compacting on the GPU against the page oracle, and together with the caches that live in the
pages."""
import numpy as np
import pytest

from oracle.pages_oracle import Pool

import helpers as H
import helpers8 as H8

pytestmark = pytest.mark.gpu


class Dev:
    """An oracle's state on the GPU.  Arrays of several widths: 16-byte pages, odd multiples of 4 bytes, more than one piece."""

    def __init__(self, oracle, longest=64):
        import torch
        self.o, self.L = oracle, H.lib()
        self.table, self.lens, self.refs = (torch.tensor(x, device="cuda") for x in (oracle.table, oracle.lens, oracle.refs))
        self.arrays = [torch.tensor(a, device="cuda") for a in oracle.arrays]
        self.ctx = self.L.lorc_create(1, 64, 1, 1, 64, 10000.0, max_pos=16)
        self.pages = self.L.make_pages(self.arrays, self.table, self.lens, self.refs, oracle.page_size)
        need = self.L.lorc_pages_workspace_bytes(self.pages, longest)
        self.ws = torch.full((need + 256,), 0x5a, dtype=torch.uint8, device="cuda")
        self.need = need
        self.L.lorc_set_workspace(self.ctx, self.ws, need)

    def ints(self, x):
        import torch
        return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")

    def call(self, what, *lists, **more):
        lists = [self.ints(x) for x in lists]
        n = [] if what == "grow" else [lists[0].numel()]
        getattr(self.L, "lorc_pages_" + what)(self.ctx, self.pages, *lists, *n, **more)
        bad = getattr(self.o, what)(*[x.cpu().numpy() for x in lists])
        self.same(bad)

    def same(self, bad=()):
        rc = self.L.lorc_sync_status(self.ctx)
        codes = {"arg": self.L.LORC_ERR_ARG, "capacity": self.L.LORC_ERR_CAPACITY}
        assert rc in {codes[b] for b in bad} if bad else rc == 0, (rc, bad)
        assert np.array_equal(self.lens.cpu().numpy(), self.o.lens)
        assert np.array_equal(self.refs.cpu().numpy(), self.o.refs)
        assert np.array_equal(self.table.cpu().numpy(), self.o.table)
        for a, want in zip(self.arrays, self.o.arrays):
            assert np.array_equal(a.cpu().numpy(), want)
        assert bool((self.ws[self.need:] == 0x5a).all())

    def close(self):
        self.L.lorc_destroy(self.ctx)


def pool(rng, rows, pages, per, ps, arrays=3):
    widths = [4, 257, 2500, 1024, 1, 36]
    return Pool(np.full((rows, per), -7, np.int32), np.zeros(rows, np.int32), np.zeros(pages, np.int32),
                [rng.integers(-2 ** 31, 2 ** 31, (pages, widths[i % 6])).astype(np.int32) for i in range(arrays)], ps)


@pytest.mark.parametrize("rows,pages,per,ps,arrays", [(6, 40, 8, 4, 3), (40, 500, 16, 16, 6), (1, 1, 1, 1, 1), (50, 9000, 300, 1, 2),
                                                      (1500, 5000, 4, 16, 1), (5, 30, 7, 3, 131), (9, 64, 8, 48, 0)])
def test_a_life_of_a_pool(rows, pages, per, ps, arrays):
    rng = np.random.default_rng([rows, pages])
    d = Dev(pool(rng, rows, pages, per, ps, arrays), longest=3 * rows + 5)
    room = rng.integers(0, max(2, per * ps // 2), rows) * (rng.random(rows) < 0.6)
    d.call("grow", room)
    for _ in range(25):
        what = rng.integers(4)
        if what == 0:
            # (with rows that are listed twice, and ones outside the table)
            d.call("free", rng.integers(-1, rows + 1, rng.integers(1, max(2, rows // 2) + 1)))
        elif what == 1:
            n = int(rng.integers(1, 2 * rows + 2))
            d.call("fork", rng.integers(-1, rows + 1, n), rng.integers(-1, rows + 1, n))
        elif what == 2:
            d.call("grow", rng.integers(-2, 2 * ps + 1, rows))
        else:
            n_used = d.ints([0])
            d.L.lorc_pages_compact(d.ctx, d.pages, n_used=n_used)
            assert d.o.compact() == int(n_used)
            d.same()
    d.close()


def test_compact_into_other_tables():
    import torch
    rng = np.random.default_rng(3)
    d = Dev(pool(rng, 30, 6000, 200, 2, 3))
    d.call("grow", rng.integers(50, 400, 30))
    d.call("free", rng.permutation(30)[:17])
    table, refs, lens = d.table.clone(), d.refs.clone(), d.lens.clone()
    before = [a.clone() for a in d.arrays]
    t_out, r_out, n = torch.full_like(table, 5), torch.full_like(refs, 5), d.ints([0])
    for _ in range(2):                       # the old tables are still what they were: the same again
        d.L.lorc_pages_compact(d.ctx, d.pages, t_out, r_out, n)
        torch.cuda.synchronize()
        assert torch.equal(d.table, table) and torch.equal(d.refs, refs) and torch.equal(d.lens, lens)
    assert d.o.compact() == int(n)
    assert np.array_equal(t_out.cpu().numpy(), d.o.table) and np.array_equal(r_out.cpu().numpy(), d.o.refs)
    for a, b, want in zip(d.arrays, before, d.o.arrays):
        assert np.array_equal(a.cpu().numpy(), want)
        used = refs > 0
        assert torch.equal(a[used], b[used])         # the old pages keep their contents
    d.close()


def test_lengths_and_entries_that_do_not_fit():
    rng = np.random.default_rng(4)
    d = Dev(pool(rng, 6, 40, 4, 4, 2))
    d.call("grow", [10, 7, 0, 0, 17, 16])            # 17 tokens do not fit four pages of four
    d.o.lens[1] = 1000
    d.lens[1] = 1000
    d.call("fork", [1, 0], [2, 3])                   # neither does that parent
    d.call("grow", [0, 1, 0, 2 ** 31 - 1, 0, 0])
    d.call("free", [1])
    d.o.table[0, 1] = 99
    d.table[0, 1] = 99
    d.call("free", [0])
    d.close()


def test_too_few_pages():
    rng = np.random.default_rng(5)
    d = Dev(pool(rng, 8, 10, 6, 4, 2))
    d.call("grow", [5, 9, 0, 0, 0, 0, 0, 0])
    d.call("fork", [0, 1, 0, 1, 1, 1], [2, 3, 4, 5, 6, 7])       # five pages are free
    d.call("grow", [8, 1, 1, 1, 1, 1, 1, 1])
    d.call("free", [3, 4, 3])
    d.call("grow", [8, 8, 0, 8, 1, 0, 0, 0])
    d.close()


def test_refusals():
    import torch
    rng = np.random.default_rng(6)
    d = Dev(pool(rng, 4, 20, 4, 4, 2))
    L = d.L
    rows = d.ints([0, 1])

    def refused(code, call, *a):
        with pytest.raises(L.LorcError) as e:
            call(d.ctx, *a)
        assert e.value.code == code, str(e.value)

    def bad(**over):
        p = L.make_pages(d.arrays, d.table, d.lens, d.refs, 4)
        p.keep = p.bufs
        for k, v in over.items():
            setattr(p, k, v)
        return p

    for p in (bad(page_table=None), bad(seq_lens=None), bad(refs=None), bad(n_pages=0), bad(page_size=0), bad(n_rows=0),
              bad(max_pages_per_seq=-1), bad(n_bufs=-1), bad(n_bufs=L.LORC_PAGES_MAX_BUFS + 1), bad(refs=d.refs.data_ptr() + 2)):
        refused(L.LORC_ERR_ARG, L.lorc_pages_free, p, rows, 2)
        refused(L.LORC_ERR_ARG, L.lorc_pages_fork, p, rows, rows, 2)
        refused(L.LORC_ERR_ARG, L.lorc_pages_grow, p, rows)
        refused(L.LORC_ERR_ARG, L.lorc_pages_compact, p)
    good = bad()
    for n in (-1, L.LORC_PAGES_MAX_LIST + 1):
        refused(L.LORC_ERR_ARG, L.lorc_pages_free, good, rows, n)
    refused(L.LORC_ERR_ARG, L.lorc_pages_free, good, None, 2)
    refused(L.LORC_ERR_ARG, L.lorc_pages_fork, good, rows, None, 2)
    refused(L.LORC_ERR_ARG, L.lorc_pages_grow, good, None)
    for size in (0, -4, 6, 2 ** 33):
        p = bad()
        p.bufs[1].page_bytes = size
        refused(L.LORC_ERR_ARG, L.lorc_pages_compact, p)
    p = bad()
    p.bufs[0].base = d.arrays[0].data_ptr() + 2
    refused(L.LORC_ERR_ARG, L.lorc_pages_fork, p, rows, rows, 2)
    refused(L.LORC_ERR_WORKSPACE, L.lorc_pages_fork, good, rows, rows, L.LORC_PAGES_MAX_LIST)
    L.lorc_set_workspace(d.ctx, None)
    refused(L.LORC_ERR_WORKSPACE, L.lorc_pages_grow, good, d.ints([0] * 4))
    L.lorc_set_workspace(d.ctx, d.ws, d.need)
    L.lorc_pages_free(d.ctx, good, None, 0)          # an empty list needs nothing
    L.lorc_pages_fork(d.ctx, good, None, None, 0)
    d.same()
    d.close()


@pytest.mark.parametrize("kind", H8.KINDS)
def test_forked_sequences_decode_apart(kind):
    """A search over continuations as a program runs it: two sequences in an 8-bit cache, three children, every one decodes
    tokens of its own (grow, write, attention), one is freed, the pool is compacted; the attention is always that of the numbers
    that a copy of the whole sequence would hold."""
    import torch
    c = H8.Case(kind, 8, 2, 128, [37, 64, 0, 0, 0], page=16, D=256, seed=21, max_len=96)
    L = c.L
    n_pages = 80
    c.kv = torch.cat([c.kv, torch.zeros(2, n_pages - c.kv.shape[1], 16, c.n, dtype=torch.int8, device="cuda")], 1).contiguous()
    c.sc = torch.cat([c.sc, torch.zeros(2, n_pages - c.sc.shape[1], 1, c.H_kv, device="cuda")], 1).contiguous()
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs[c.table[0, :3].long()] = 1
    refs[c.table[1, :4].long()] = 1
    pages = L.make_pages([c.kv[0], c.kv[1], c.sc[0], c.sc[1]], c.table, c.sl, refs, 16)
    need = max(L.lorc_pages_workspace_bytes(pages, 8), L.lorc_cache8_workspace_bytes(c.ctx, 5, 96, 1))
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    L.lorc_set_workspace(c.ctx, ws)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731

    # a second cache in which every sequence has pages of its own
    alone = H8.Case(kind, 8, 2, 128, [37, 64, 37, 64, 37], page=16, D=256, seed=21, max_len=96)
    alone.workspace(1)
    for s, a in enumerate([0, 1, 0, 1, 0]):
        for j in range(4):
            alone.kv[:, alone.table[s, j]] = c.kv[:, c.table[a, j]]
            alone.sc[:, alone.table[s, j]] = c.sc[:, c.table[a, j]]
    L.lorc_pages_fork(c.ctx, pages, i32([0, 1, 0]), i32([2, 3, 4]), 3)
    live = [0, 1, 2, 3, 4]
    for step in range(12):
        if step == 7:
            L.lorc_pages_free(c.ctx, pages, i32([1]), 1)
            live.remove(1)
        if step in (5, 9):
            L.lorc_pages_compact(c.ctx, pages)
        room = i32([1 if s in live else 0 for s in range(5)])
        L.lorc_pages_grow(c.ctx, pages, room)
        alone.sl += 1
        x = torch.randn(5, 1, 256, device="cuda").bfloat16()
        q = torch.randn(5, 8, 128, device="cuda").bfloat16()
        outs = []
        for e in (c, alone):
            out = torch.zeros(5, 8, 128, dtype=torch.bfloat16, device="cuda")
            cache = e.cache(n_pages=e.kv.shape[1])
            L.lorc_append8(e.ctx, 0, cache, x)
            L.lorc_decode_attn8(e.ctx, 0, cache, q, out)
            outs.append(out)
        if len(live) == 5:
            assert c.status() == 0
        else:
            assert c.status() in (L.LORC_ERR_EMPTY, L.LORC_ERR_CAPACITY)      # (the freed row: nothing to write to, nothing to attend to)
        assert alone.status() == 0
        assert torch.equal(outs[0][live], outs[1][live]), step
    held = torch.zeros_like(refs)
    for s in live:
        held.index_add_(0, c.table[s, : -(-int(c.sl[s]) // 16)].long(), torch.ones_like(c.table[s, : -(-int(c.sl[s]) // 16)]))
    assert torch.equal(held, refs)
    c.close()
    alone.close()


def test_a_captured_search_step():
    import torch
    rng = np.random.default_rng(8)
    d = Dev(pool(rng, 10, 200, 20, 4, 3))
    d.call("grow", [30, 41, 0, 0, 0, 0, 0, 0, 0, 0])
    parents, kids = d.ints([0, 1, 1, 0]), d.ints([2, 3, 4, 5])
    room = d.ints([0, 0, 1, 1, 1, 1, 0, 0, 0, 0])

    def step():
        d.L.lorc_pages_free(d.ctx, d.pages, kids, 4)
        d.L.lorc_pages_fork(d.ctx, d.pages, parents, kids, 4)
        d.L.lorc_pages_grow(d.ctx, d.pages, room)

    def oracle():
        d.o.free(kids.cpu().numpy())
        d.o.fork(parents.cpu().numpy(), kids.cpu().numpy())
        d.o.grow(room.cpu().numpy())

    step()
    oracle()
    d.same()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(3):
        graph.replay()
        oracle()
        torch.cuda.synchronize()
        d.same()
    parents.copy_(d.ints([1, 1, 1, 1]))
    graph.replay()
    oracle()
    torch.cuda.synchronize()
    d.same()
    d.close()
