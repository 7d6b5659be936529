"""What forking, growing, freeing and compacting have to keep, checked on the page oracle itself; and what the library
refuses without a GPU."""
import numpy as np
import pytest

from oracle.pages_oracle import Pool

import helpers as H


def random_pool(rng, rows=12, pages=64, per=8, ps=4, live=5):
    p = Pool(np.full((rows, per), -1, np.int32), np.zeros(rows, np.int32), np.zeros(pages, np.int32),
             [rng.integers(0, 1000, (pages, 3))], ps)
    room = np.zeros(rows, np.int32)
    room[rng.permutation(rows)[:live]] = rng.integers(1, per * ps // 2, live)
    p.grow(room)
    return p


def tokens(p, r):
    return [tuple(p.arrays[0][page]) for page in p.table[r, :p.held(p.lens[r])]]


def counts(p):
    n = np.zeros_like(p.refs)
    for r in range(len(p.lens)):
        np.add.at(n, p.table[r, :p.held(p.lens[r])], 1)
    return n


@pytest.mark.parametrize("seed", range(8))
def test_a_life_of_a_pool(seed):
    rng = np.random.default_rng(seed)
    p = random_pool(rng)
    for _ in range(30):
        what = rng.integers(4)
        before = {r: (int(p.lens[r]), tokens(p, r)) for r in range(len(p.lens))}
        if what == 0:
            rows = rng.permutation(len(p.lens))[:rng.integers(0, 4)]
            p.free(rows)
            changed = set(rows)
        elif what == 1:
            empty = np.flatnonzero(p.lens == 0)
            kids = rng.permutation(empty)[:4]
            parents = rng.integers(0, len(p.lens), len(kids))
            p.fork(parents, kids)
            changed = set(kids)
            for a, c in zip(parents, kids):
                if p.lens[c]:
                    assert p.lens[c] == before[a][0] and tokens(p, c) == before[a][1]
                    last = p.held(p.lens[c]) - 1
                    if p.lens[c] % p.page_size:
                        assert p.table[c, last] != p.table[a, last] and p.refs[p.table[c, last]] == 1
        elif what == 2:
            room = rng.integers(-2, 3, len(p.lens))
            p.grow(room)
            changed = set(np.flatnonzero(room > 0))
        else:
            n = p.compact()
            assert (p.refs[:n] > 0).all() and not p.refs[n:].any()
            changed = set()
        assert np.array_equal(counts(p), p.refs)
        for r, (n, t) in before.items():
            if r not in changed:
                assert p.lens[r] == n and tokens(p, r) == t


def test_workspace_and_null_arguments_without_a_gpu():
    b = H.lib()
    import ctypes
    p = b.lorc_pages(None, 0, 100, 16, 8, 4, 0, None, None, None)
    assert b.lorc_pages_workspace_bytes(p, 10) > 100 * 4
    assert b.lorc_pages_workspace_bytes(p, -1) == 0 and b.lorc_pages_workspace_bytes(p, b.LORC_PAGES_MAX_LIST + 1) == 0
    for field in ("n_pages", "page_size", "max_pages_per_seq", "n_rows"):
        q = b.lorc_pages(None, 0, 100, 16, 8, 4, 0, None, None, None)
        setattr(q, field, 0)
        assert b.lorc_pages_workspace_bytes(q, 10) == 0
    q.n_rows, q.n_bufs = 4, b.LORC_PAGES_MAX_BUFS + 1
    assert b.lorc_pages_workspace_bytes(q, 10) == 0
    lib = b._lib
    assert lib.lorc_pages_workspace_bytes(None, 1) == 0
    assert lib.lorc_cache8_workspace_bytes(None, 1, 1, 1) == 0
    c = b.lorc_cache8()
    for call in (lambda: lib.lorc_append8(None, 0, ctypes.byref(c), None, 1, None),
                 lambda: lib.lorc_decode_attn8(None, 0, ctypes.byref(c), None, None, None),
                 lambda: lib.lorc_prefill_attn8(None, 0, ctypes.byref(c), None, None, 1, None),
                 lambda: lib.lorc_pages_free(None, ctypes.byref(p), None, 1, None),
                 lambda: lib.lorc_pages_fork(None, ctypes.byref(p), None, None, 1, None),
                 lambda: lib.lorc_pages_grow(None, ctypes.byref(p), None, None),
                 lambda: lib.lorc_pages_compact(None, ctypes.byref(p), None, None, None, None)):
        assert call() == b.LORC_ERR_ARG
    assert ctypes.sizeof(b.lorc_cache8) == 6 * 8 + 6 * 4 + 8 and b.lorc_cache8.seq_stride.offset == 72
    assert ctypes.sizeof(b.lorc_pages) == 8 + 6 * 4 + 3 * 8 and ctypes.sizeof(b.lorc_page_buf) == 16


def test_make_pages_checks_its_tensors():
    import torch
    b = H.lib()
    t, lens, refs = torch.zeros(3, 5, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(7, dtype=torch.int32)
    pool = torch.zeros(7, 16, 24, dtype=torch.bfloat16)
    p = b.make_pages([pool], t, lens, refs, 16)
    assert (p.n_pages, p.max_pages_per_seq, p.n_rows, p.n_bufs, p.bufs[0].page_bytes) == (7, 5, 3, 1, 16 * 24 * 2)
    for bad in (lambda: b.make_pages([pool[:6]], t, lens, refs, 16), lambda: b.make_pages([pool[:, :, :8]], t, lens, refs, 16),
                lambda: b.make_pages([pool], t.long(), lens, refs, 16), lambda: b.make_pages([pool], t, lens[:2], refs, 16),
                lambda: b.make_pages([pool], t, lens.float(), refs, 16), lambda: b.make_pages([pool], t[:, ::2], lens, refs, 16)):
        with pytest.raises(ValueError):
            bad()
