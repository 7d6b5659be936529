"""The 8-bit cache of uncompressed layers against its fp64 restatement: cache write, decode attention, prompt chunks."""
import numpy as np
import pytest

from oracle import cache8_oracle as C8

import helpers as H
import helpers8 as H8

pytestmark = pytest.mark.gpu


def _decode(c, scale=2.0, **over):
    import torch
    q, qd = c.queries(scale=scale)
    out = torch.full((c.b, c.H_q, c.d_h), 7.0, dtype=torch.bfloat16, device="cuda")
    c.workspace()
    c.L.lorc_decode_attn8(c.ctx, 0, c.cache(**over), qd, out)
    return q, H.host_f64(out).reshape(c.b, 1, c.H_q, c.d_h)


GEOMETRIES = [(4, 2, 64), (32, 8, 128), (8, 1, 128), (3, 3, 128), (21, 3, 64), (5, 5, 64), (12, 6, 128)]


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("heads", GEOMETRIES)
@pytest.mark.parametrize("lens,page", [([1], 0), ([17, 1, 64, 63], 16), ([255, 256, 257, 65], 0), ([777, 16, 300], 48), ([1030, 129], 64)])
def test_decode(kind, heads, lens, page):
    c = H8.Case(kind, *heads, lens, page=page, seed=len(lens))
    q, got = _decode(c)
    H8.assert_attention(got, *c.want(q))
    assert c.status() == 0 and c.guard_intact()
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("style", [0, 1, 2])
@pytest.mark.parametrize("d_h", [64, 128])
def test_decode_rotations_and_peaked_scores(kind, style, d_h):
    c = H8.Case(kind, 8, 2, d_h, [900, 333], page=32, style=style, theta=500000.0, seed=style)
    for scale in (0.01, 1.0, 16.0):
        q, got = _decode(c, scale)
        H8.assert_attention(got, *c.want(q))
    assert c.status() == 0
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
def test_decode_long_and_ragged(kind):
    """Few long sequences (many parts each), and many lengths at once (parts that begin and end inside sequences)."""
    rng = np.random.default_rng(5)
    for lens, page in (([8000], 0), ([5000, 8, 2500, 1], 64), (list(rng.integers(1, 900, 70)), 128)):
        c = H8.Case(kind, 8, 2, 128, lens, page=page, seed=len(lens))
        q, got = _decode(c)
        H8.assert_attention(got, *c.want(q))
        assert c.status() == 0 and c.guard_intact()
        c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("heads,b,page", [((16, 8, 128), 90, 0), ((8, 8, 64), 170, 64), ((4, 1, 128), 400, 16)])
def test_decode_of_many_short_sequences(kind, heads, b, page):
    """More sequences than blocks, none longer than 256 tokens, some empty."""
    rng = np.random.default_rng(b)
    lens = [int(x) for x in rng.integers(1, 257, b)]
    for s in (0, 1, 40, b - 1):
        lens[s] = 0
    lens[2], lens[3] = 256, 1
    c = H8.Case(kind, *heads, lens, page=page, seed=b)
    q, got = _decode(c)
    H8.assert_attention(got, *c.want(q))
    assert not got[[0, 1, 40, b - 1]].any() and c.status() == c.L.LORC_ERR_EMPTY and c.guard_intact()
    c.close()


def test_decode_of_many_sequences():
    """More sequences than one look at the lengths covers, with parts that begin and end inside them, and empty ones among them."""
    rng = np.random.default_rng(6)
    lens = [int(x) for x in rng.integers(1, 600, 170)]
    for heads in ((4, 1, 64), (8, 8, 64)):
        c = H8.Case("int8", *heads, lens, page=16, D=64, seed=60, max_len=600)
        q, got = _decode(c)
        want = c.want(q)
        H8.assert_attention(got, *want)
        assert c.status() == 0 and c.guard_intact()
        import torch
        for s in (0, 31, 32, 128, 150, 169):
            c.lens[s] = 0
            for w in want:
                w[s] = 0.0
        c.sl.copy_(torch.tensor(c.lens, dtype=torch.int32))
        out = torch.full((c.b, c.H_q, c.d_h), 7.0, dtype=torch.bfloat16, device="cuda")
        c.L.lorc_decode_attn8(c.ctx, 0, c.cache(), H.dev_bf16(q[:, 0]), out)
        H8.assert_attention(H.host_f64(out).reshape(got.shape), *want)
        assert c.status() == c.L.LORC_ERR_EMPTY
        c.close()


def test_a_pool_beyond_32_bit_offsets():
    """Pages more than 2^32 bytes into a pool: write, both attentions, fork and compaction reach them."""
    import torch
    L = H.lib()
    n_pages, ps, n = 36000, 128, 1024
    kv = torch.zeros(2, n_pages, ps, n, dtype=torch.int8, device="cuda")
    sc = torch.zeros(2, n_pages, ps // 16, 8, device="cuda")
    small = H8.Case("int8", 32, 8, 128, [300, 140], page=ps, D=256, seed=61)
    far = torch.tensor([[n_pages - 1, n_pages - 7, n_pages - 3], [n_pages - 2, n_pages - 9, n_pages - 4]], dtype=torch.int32, device="cuda")
    kv[:, far.flatten().long()] = small.kv[:, small.table.flatten().long()]
    sc[:, far.flatten().long()] = small.sc[:, small.table.flatten().long()]
    cache = L.make_cache8(kv[0], kv[1], sc[0], sc[1], small.sl, 2, 300, L.LORC_CACHE8_INT8, page_table=far, page_size=ps,
                          max_pages_per_seq=3, n_pages=n_pages)
    small.workspace(100)
    x = H.dev_bf16(small.rng.standard_normal((2, 100, 256)))
    q = H.dev_bf16(small.rng.standard_normal((2, 100, 32, 128)))
    outs = []
    for c in (small.cache(), cache):
        out, dec = torch.zeros_like(q), torch.zeros(2, 32, 128, dtype=torch.bfloat16, device="cuda")
        L.lorc_append8(small.ctx, 0, c, x, 100)
        L.lorc_append8(small.ctx, 0, c, x[:, 99:].contiguous(), 1)
        L.lorc_prefill_attn8(small.ctx, 0, c, q, out, 100)
        L.lorc_decode_attn8(small.ctx, 0, c, q[:, 0].contiguous(), dec)
        outs.append((out, dec))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    assert torch.equal(kv[:, far.flatten().long()], small.kv[:, small.table.flatten().long()])
    assert small.status() == 0
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs[far.flatten().long()] = 1
    table = torch.cat([far, torch.full_like(far, -1)])
    lens = torch.tensor([300, 384, 0, 0], dtype=torch.int32, device="cuda")
    pages = L.make_pages([kv[0], kv[1], sc[0], sc[1]], table, lens, refs, ps)
    ws = torch.zeros(L.lorc_pages_workspace_bytes(pages, 2), dtype=torch.uint8, device="cuda")
    L.lorc_set_workspace(small.ctx, ws)
    want = [kv[:, far[0].long()].clone(), sc[:, far[1].long()].clone()]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    L.lorc_pages_fork(small.ctx, pages, i32([0]), i32([2]), 1)
    assert int(table[2, 2]) == 0 and torch.equal(kv[:, 0], kv[:, n_pages - 3])
    L.lorc_pages_compact(small.ctx, pages)
    assert torch.equal(kv[:, table[0].long()], want[0]) and torch.equal(sc[:, table[1].long()], want[1])
    assert int(table.max()) == 6 and small.status() == 0
    small.close()


@pytest.mark.parametrize("kind", H8.KINDS)
def test_the_debug_flag_keeps_the_results(kind):
    """The plain projection and the attention off the tcgen05 kernels: within the same bounds."""
    import torch
    c = H8.Case(kind, 32, 8, 128, [130, 517], page=64, seed=62, flags=H.lib().LORC_FLAG_DEBUG_FP32, style=H.ROPE_NONE)
    at, x = _exact_x(c, 130)
    c.workspace(130)
    c.L.lorc_append8(c.ctx, 0, c.cache(), x, 130)
    assert c.L.lorc_last_path(c.ctx) == 1
    c.codes, c.scales = H8.host_codes(c.kv, kind), c.sc.double().cpu().numpy()
    for s, n in enumerate(c.lens):
        new = np.asarray(c.w[1], dtype=np.float64)[at[s]].reshape(130, c.H_kv, c.d_h)
        page, row = c.rows_of(s, n)
        step = c.scales[1][page, row // 16][n - 130:][..., None]
        assert (np.abs(c.held(1, s, n)[n - 130:] - new) <= (step / 2 if kind == "int8" else np.maximum(2.0 ** -4 * np.abs(new), step * 2.0 ** -10))).all()
    q, qd = c.queries(130, scale=1.0)
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda")
    c.L.lorc_prefill_attn8(c.ctx, 0, c.cache(), qd, out, 130)
    assert c.L.lorc_last_path(c.ctx) == 3
    H8.assert_attention(H.host_f64(out), *c.want(q, 130))
    assert c.status() == 0
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
def test_decode_scales_of_any_size(kind):
    """Scales that are no powers of two, differ by 2^40 between blocks, or are zero."""
    c = H8.Case(kind, 8, 2, 128, [700, 90], seed=3)
    c.scales = np.abs(c.rng.standard_normal(c.scales.shape)) * 1e-2
    c.scales[1] *= np.ldexp(1.0, c.rng.integers(-40, 1, c.scales[1].shape))
    c.scales[:, :, 2] = 0.0
    c.scales = c.scales.astype(np.float32).astype(np.float64)
    c.upload()
    q, got = _decode(c)
    H8.assert_attention(got, *c.want(q))
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("block", [0, 3, 6])
def test_small_values_beside_large_ones_of_little_weight(kind, block):
    """One block has values 2^22 times as large as all others, and scores far below theirs: the weights of the small values keep
    their precision.  With B the average of max|v_i|: weights as fp16 numbers are off by 2^-11 of themselves, or, where they are below
    2^-14 of the largest one, by 2^-25 of that one, whose token has a code above a third of the largest (checked here): N tokens together by
    (2^-11 + 3 N 2^-25) B.  Scores as in assert_attention, which gives 2^-15 (1 + A) B."""
    import torch
    c = H8.Case(kind, 4, 2, 64, [100, 112], style=2, seed=20 + block)
    largest = 127 if kind == "int8" else 448
    for score in (4.0, 9.0, 14.0, 16.0, 25.0):
        q = H.synth.to_bf16_exact(np.repeat(c.rng.standard_normal((c.b, 1, c.H_kv, c.d_h)), c.G, axis=2)).astype(np.float64)
        c.scales[0] = 2.0 ** -9 if kind == "int8" else 2.0 ** -11
        c.scales[1] = 2.0 ** -24
        for s in range(c.b):
            for h in range(c.H_kv):
                x = q[s, 0, h * c.G]
                unit = C8.round_code(-x / np.abs(x).max() * largest, kind)
                c.codes[0][s, 16 * block:16 * block + 16, h * c.d_h:(h + 1) * c.d_h] = unit
                c.scales[0][s, block, h] = np.float32(score * np.sqrt(c.d_h) / -(unit @ x))
                c.scales[1][s, block, h] = 2.0 ** -2
        c.upload()
        qd = H.dev_bf16(q)
        out = torch.zeros(c.b, c.H_q, c.d_h, dtype=torch.bfloat16, device="cuda")
        c.workspace()
        c.L.lorc_decode_attn8(c.ctx, 0, c.cache(), qd, out)
        got = H.host_f64(out)
        want, size, _ = c.want(q)
        for s, n in enumerate(c.lens):
            k, v = c.held(0, s, n), c.held(1, s, n)
            assert (np.abs(c.codes[1][s, :n].reshape(n, c.H_kv, c.d_h)).max(-1) > largest / 3).all()
            for h in range(c.H_q):
                x = k[:, h // c.G] @ q[s, 0, h] / np.sqrt(c.d_h)
                w = np.exp(x - x.max())
                B = (w * np.abs(v[:, h // c.G]).max(-1)).sum() / w.sum()
                bound = 2.0 ** -8 * np.abs(want[s, 0, h]) + (2.0 ** -11 + 3 * n * 2.0 ** -25 + 2.0 ** -15 * (1 + size[s, 0, h])) * B
                assert (np.abs(got[s, h] - want[s, 0, h]) <= bound).all(), (score, s, h)
    assert c.status() == 0
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("T", [1, 5])
def test_rows_behind_the_end_are_not_read(kind, T):
    """Whatever stands behind a sequence's end: codes of NaN, scales that are NaN or infinite."""
    import torch
    c = H8.Case(kind, 32, 8, 128, [77, 5, 600], page=64, seed=4)
    q, qd = c.queries(T)
    c.workspace(T)
    out = torch.zeros(c.b, T, c.H_q, c.d_h, dtype=torch.bfloat16, device="cuda")
    call = (lambda: c.L.lorc_decode_attn8(c.ctx, 0, c.cache(), qd, out)) if T == 1 else \
        (lambda: c.L.lorc_prefill_attn8(c.ctx, 0, c.cache(), qd, out, T))
    call()
    want = out.clone()
    held = np.zeros(c.codes.shape[1:3], dtype=bool)
    for s, n in enumerate(c.lens):
        held[c.rows_of(s, n)] = True
    dead = torch.from_numpy(~held).cuda()
    c.kv[:, dead] = 0x7f
    c.sc[:, torch.from_numpy(~held.reshape(held.shape[0], -1, 16).any(-1)).cuda()] = float("nan")
    out.zero_()
    call()
    assert torch.equal(out, want)
    H8.assert_attention(H.host_f64(out), *c.want(q, T), fp16=T > 1)
    assert c.status() == 0
    c.close()


def test_empty_and_overlong_sequences():
    import torch
    c = H8.Case("int8", 8, 2, 128, [300, 0, 40], seed=6)
    q, got = _decode(c)
    H8.assert_attention(got, *c.want(q))
    assert not got[1].any() and c.status() == c.L.LORC_ERR_EMPTY and c.status() == 0
    # a length beyond max_seq_len: reported, zeros, the others as before
    c.lens = [300, 0, 40]
    c.sl.copy_(torch.tensor([300, 10 ** 6, 40], dtype=torch.int32))
    q, got = _decode(c)
    H8.assert_attention(got, *c.want(q))
    assert not got[1].any() and c.status() == c.L.LORC_ERR_CAPACITY
    c.close()


@pytest.mark.parametrize("lens", [[200, 100], [2000, 300]])
def test_pages_outside_the_pool_are_left_out(lens):
    import torch
    c = H8.Case("e4m3", 8, 2, 128, lens, page=32, seed=7)
    q, qd = c.queries()
    c.table[0, 2] = -1
    c.table[1, 1] = 10 ** 6
    c.workspace()
    out = torch.zeros(c.b, c.H_q, c.d_h, dtype=torch.bfloat16, device="cuda")
    c.L.lorc_decode_attn8(c.ctx, 0, c.cache(), qd, out)
    assert c.status() == c.L.LORC_ERR_CAPACITY
    got = H.host_f64(out)
    for s, gone in ((0, 2), (1, 1)):
        keep = np.arange(c.lens[s]) // 32 != gone
        k, v = c.held(0, s, c.lens[s])[keep], c.held(1, s, c.lens[s])[keep]
        want, size = C8.attention(k, v, c.rotate(q[s, 0], c.lens[s] - 1), c.G)
        H8.assert_attention(got[s], want, size[:, None], np.repeat(np.abs(v).max(axis=(0, 2)), c.G)[:, None])
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("heads,fp16", [((32, 8, 128), True), ((64, 8, 128), True), ((4, 2, 64), False), ((6, 2, 128), False)])
@pytest.mark.parametrize("T,lens,page", [(2, [2, 40], 0), (31, [31, 64, 200], 16), (130, [130, 517], 64)])
def test_prompt_chunks(kind, heads, fp16, T, lens, page):
    import torch
    c = H8.Case(kind, *heads, lens, page=page, seed=T)
    q, qd = c.queries(T, scale=1.0)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    c.workspace(T)
    c.L.lorc_prefill_attn8(c.ctx, 0, c.cache(), qd, out, T)
    H8.assert_attention(H.host_f64(out), *c.want(q, T), fp16=fp16)
    assert c.status() == 0 and c.guard_intact()
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("T,lens,page", [(40, [5000], 0), (70, [70, 2500, 1000], 64), (33, [33, 40, 4000], 16)])
def test_chunks_behind_long_contexts(kind, T, lens, page):
    """Few queries and many keys: CTAs share the keys of a block of queries, and some have none of a short sequence's."""
    import torch
    c = H8.Case(kind, 32, 8, 128, lens, page=page, seed=T)
    q, qd = c.queries(T, scale=1.0)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    c.workspace(T)
    c.L.lorc_prefill_attn8(c.ctx, 0, c.cache(), qd, out, T)
    assert c.L.lorc_last_path(c.ctx) == 2
    H8.assert_attention(H.host_f64(out), *c.want(q, T), fp16=True)
    assert c.status() == 0 and c.guard_intact()
    # a sequence that is shorter than the chunk, and one without tokens
    if len(lens) == 3:
        c.lens = [T - 1, lens[1], 0]
        c.sl.copy_(torch.tensor(c.lens, dtype=torch.int32))
        c.L.lorc_prefill_attn8(c.ctx, 0, c.cache(), qd, out, T)
        H8.assert_attention(H.host_f64(out), *c.want(q, T), fp16=True)
        assert not out[0].any() and not out[2].any() and c.status() in (c.L.LORC_ERR_ARG, c.L.LORC_ERR_EMPTY)
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("heads", [(4, 2, 64), (8, 8, 128), (6, 2, 128), (32, 8, 128), (10, 2, 64), (8, 1, 64)])
@pytest.mark.parametrize("T,lens,page", [(2, [2, 3, 64, 65, 250], 0), (3, [1500, 3, 700], 48), (5, [129, 128, 2003, 5], 64),
                                         (9, list(range(9, 400, 17)), 16)])
def test_few_queries(kind, heads, T, lens, page):
    """Queries that share a pass over their sequence, each with its own last token, with parts that begin and end inside
    sequences; T of them, and, with the same workspace, fewer."""
    import torch
    c = H8.Case(kind, *heads, lens, page=page, style=T % 2, theta=500000.0, seed=T, flags=H.lib().LORC_FLAG_DEBUG_FP32)
    c.workspace(T)
    for t in (T, T - 1):
        q, qd = c.queries(t, scale=2.0)
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        c.L.lorc_prefill_attn8(c.ctx, 0, c.cache(), qd, out, t)
        assert c.L.lorc_last_path(c.ctx) == 3
        H8.assert_attention(H.host_f64(out), *c.want(q, t))
        assert c.status() == 0 and c.guard_intact()
    c.close()


@pytest.mark.parametrize("heads", [(32, 8, 128), (4, 2, 64)])
def test_a_chunk_longer_than_a_sequence(heads):
    import torch
    c = H8.Case("int8", *heads, [50, 7, 0], seed=8)
    q, qd = c.queries(20, scale=1.0)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    c.workspace(20)
    c.L.lorc_prefill_attn8(c.ctx, 0, c.cache(), qd, out, 20)
    H8.assert_attention(H.host_f64(out), *c.want(q, 20), fp16=heads[2] == 128)
    assert not out[1:].any() and c.status() in (c.L.LORC_ERR_ARG, c.L.LORC_ERR_EMPTY)
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("heads", [(4, 2, 64), (8, 8, 128), (6, 2, 128), (10, 2, 64), (7, 1, 128), (3, 3, 64), (48, 8, 64)])
@pytest.mark.parametrize("T,lens,page,style", [(300, [300, 4000], 0, 1), (257, [300, 257, 700, 420, 2500], 64, 0), (150, [5000], 128, 2)])
def test_prompt_chunks_of_all_heads(kind, heads, T, lens, page, style):
    """Any number of query heads per KV head (blocks of rows that they do not fill), heads of 64, both rotations; keys shared among
    CTAs and not."""
    import torch
    c = H8.Case(kind, *heads, lens, page=page, style=style, theta=500000.0, seed=T)
    q, qd = c.queries(T, scale=1.0)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    c.workspace(T)
    c.L.lorc_prefill_attn8(c.ctx, 0, c.cache(), qd, out, T)
    assert c.status() == 0 and c.guard_intact()
    some = np.unique(np.r_[0, 1, T // 3, T - 2, T - 1, c.rng.integers(0, T, 12)])
    got = H.host_f64(out)
    want, size, vmax = c.want_some(q, T, some)
    H8.assert_attention(got[:, some], want, size, vmax, fp16=True)
    # every row has been written, from keys that it sees: rows of zeros are as unlikely as rows of sevens
    assert not (got == 7.0).all(-1).any() and not (got == 0.0).all(-1).any()
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("which", [0, 1])
def test_chunks_report_numbers_beyond_fp16(kind, which):
    """The tcgen05 path holds keys and values in fp16: up to 65504 they count, what is larger is reported."""
    import torch
    c = H8.Case(kind, 32, 8, 128, [1500, 200], seed=11)
    largest = C8.LARGEST[kind]
    c.codes[which][1, 100, 5] = largest
    fits = 2.0 ** np.floor(np.log2(65504 / largest))
    if which == 0:
        c.codes[0][1, 96:112, :128] = 0
        c.codes[0][1, 100, 5] = largest
    q, qd = c.queries(130, scale=1.0 if which else 2.0 ** -12)
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda")
    c.workspace(130)
    for scale, status in ((fits, 0), (2 * fits, c.L.LORC_ERR_ARG), (2.0 ** 100, c.L.LORC_ERR_ARG)):
        c.scales[which][1, 6, 0] = scale
        c.upload()
        c.L.lorc_prefill_attn8(c.ctx, 0, c.cache(), qd, out, 130)
        assert c.L.lorc_last_path(c.ctx) == 2 and c.status() == status
        if status == 0:
            H8.assert_attention(H.host_f64(out), *c.want(q, 130), fp16=True)
    # behind a sequence's end nothing is looked at
    c.scales[which][1, 6, 0] = 2.0 ** -6
    c.scales[which][1, 13, :] = 2.0 ** 100
    c.upload()
    c.L.lorc_prefill_attn8(c.ctx, 0, c.cache(), qd, out, 130)
    assert c.status() == 0
    c.close()


# ---- the write --------------------------------------------------------------------------------------------------------------

def _exact_x(c, T):
    """Hidden states with a single one each: the projections are rows of the weights, without rounding."""
    import torch
    at = c.rng.integers(0, c.D, (c.b, T))
    x = np.zeros((c.b, T, c.D))
    x[np.arange(c.b)[:, None], np.arange(T), at] = 1.0
    return at, H.dev_bf16(x)


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("heads,D", [((4, 2, 64), 256), ((4, 4, 128), 512), ((3, 3, 64), 200), ((3, 3, 64), 320)])
@pytest.mark.parametrize("T,lens,page", [(1, [1, 16, 17, 32, 100], 0), (1, [49, 64, 65], 16), (15, [15, 31, 47, 40], 48),
                                         (16, [16, 33], 0), (37, [37, 100, 64], 64), (300, [300, 333], 128),
                                         (20, list(range(20, 80, 2)), 16), (500, [507], 0)])
def test_write_is_exact_where_the_projection_is(kind, heads, D, T, lens, page):
    """No rotation and one-hot hidden states: codes and scales are the oracle's, bit for bit; all else stays as it was."""
    c = H8.Case(kind, *heads, lens, page=page, D=D, style=H.ROPE_NONE, seed=T)
    # weights of very different sizes, so that scales grow
    for i in range(2):
        c.w[i] = H.synth.to_bf16_exact(c.w[i] * np.ldexp(1.0, c.rng.integers(-6, 3, (D, 1))))
    c.L.lorc_load_factors(c.ctx, 0, c.L.LORC_MODE_FULL, 0, 0, H.dev_bf16(c.w[0]), None, H.dev_bf16(c.w[1]), None)
    at, x = _exact_x(c, T)
    want_codes, want_scales = c.codes.copy(), c.scales.copy()
    for s, n in enumerate(c.lens):
        page_i, row = c.rows_of(s, -(-n // 16) * 16)
        for i in range(2):
            codes = want_codes[i][page_i, row].reshape(-1, c.H_kv, c.d_h)
            scales = want_scales[i][page_i[::16], row[::16] // 16]
            C8.write(codes, scales, np.asarray(c.w[i], dtype=np.float64)[at[s]].reshape(T, c.H_kv, c.d_h), n, kind)
            want_codes[i][page_i, row] = codes.reshape(-1, c.n)
            want_scales[i][page_i[::16], row[::16] // 16] = scales
    c.workspace(T)
    for _ in range(2):                       # the same tokens again change nothing
        c.L.lorc_append8(c.ctx, 0, c.cache(), x, T)
        assert np.array_equal(c.sc.double().cpu().numpy(), want_scales)
        assert np.array_equal(H8.host_codes(c.kv, kind), want_codes)
    assert c.status() == 0 and c.guard_intact()
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("heads,D,T,lens", [((4, 2, 64), 256, 3, [3, 50]), ((8, 8, 128), 1024, 1, [100, 31, 16]),
                                            ((8, 2, 128), 512, 70, [70, 171]), ((2, 2, 64), 264, 9, [30]),
                                            ((32, 8, 128), 1024, 300, [300, 417, 355])])
def test_write_of_gaussian_tokens(kind, style, heads, D, T, lens):
    """Every new number within half a code step of the fp64 projection (and the fp32 error of the projection)."""
    c = H8.Case(kind, *heads, lens, page=32, D=D, style=style, theta=500000.0, seed=T + style)
    x = H.synth.to_bf16_exact(c.rng.standard_normal((c.b, T, D)))
    c.workspace(T)
    c.L.lorc_append8(c.ctx, 0, c.cache(), H.dev_bf16(x), T)
    assert c.status() == 0 and c.guard_intact()
    c.codes, c.scales = H8.host_codes(c.kv, kind), c.sc.double().cpu().numpy()
    x = x.astype(np.float64)
    for s, n in enumerate(c.lens):
        for i in range(2):
            w = np.asarray(c.w[i], dtype=np.float64)
            new = (x[s] @ w).reshape(T, c.H_kv, c.d_h)
            # fp32 sums of D products: 2^-16 of the sum of magnitudes; a rotation mixes two numbers and adds 2^-22 of them
            slack = 2.0 ** -16 * (np.abs(x[s]) @ np.abs(w)).reshape(T, c.H_kv, c.d_h)
            if i == 0:
                new = np.stack([c.rotate(new[t], n - T + t) for t in range(T)])
                slack = 2 * slack.max(axis=-1, keepdims=True)
            got = c.held(i, s, n)[n - T:]
            page, row = c.rows_of(s, n)
            scale = c.scales[i][page, row // 16][n - T:][..., None]
            half = scale / 2 if kind == "int8" else np.maximum(2.0 ** -4 * np.abs(new), scale * 2.0 ** -10)
            assert (np.abs(got - new) - (half + slack * (1 if kind == "int8" else 1.1)) <= 0).all()
            # the scale is the smallest that holds the block's new numbers (to the projection's error), where all are new
            for b0 in range(-(-(n - T) // 16) * 16, n, 16):
                blk = slice(b0 - (n - T), min(n, b0 + 16) - (n - T))
                most, off = np.abs(new[blk]).max(axis=(0, 2)), slack[blk].max()
                sc = scale[blk][0, :, 0]
                assert ((sc >= C8.scale_for(most - off, kind)) & (sc <= C8.scale_for(most + off, kind))).all()
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("heads,D", [((4, 2, 64), 512), ((3, 3, 128), 5120), ((7, 1, 64), 8192)])
@pytest.mark.parametrize("b", [1, 16, 37])
def test_write_of_single_tokens(kind, style, heads, D, b):
    """One token per sequence, at every place of a block: as gaussian tokens, and exactly."""
    lens = [1 + (29 * s) % 67 for s in range(b)]
    test_write_of_gaussian_tokens(kind, style, heads, D, 1, lens)
    if style == 0:
        test_write_is_exact_where_the_projection_is(kind, heads, D, 1, lens, 16)


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("heads,D", [((8, 8, 128), 512), ((17, 17, 64), 512), ((8, 8, 128), 1024), ((8, 8, 128), 8192)])
@pytest.mark.parametrize("T,lens", [(1, [1 + (29 * s) % 67 for s in range(37)]), (1, [5 + s % 40 for s in range(150)]),
                                    (3, [3 + (7 * s) % 50 for s in range(24)]), (16, [16 + s for s in range(7)]),
                                    (20, [20, 33, 47]), (70, [75])])
def test_write_of_few_tokens(kind, heads, D, T, lens):
    """Batches of decode steps, drafts and short prompts, with D split over a cluster."""
    test_write_of_gaussian_tokens(kind, T % 2, heads, D, T, lens)
    if D <= 1024:
        test_write_is_exact_where_the_projection_is(kind, heads, D, T, lens, 16 if T == 3 else 0)


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("T,lens", [(1, [17 + s % 30 for s in range(40)]), (5, [20, 40, 61, 33, 44, 25, 70, 9, 31])])
def test_finite_numbers_beside_others_in_small_batches(kind, T, lens):
    test_finite_numbers_beside_others_count_for_the_scale(kind, T, lens, path=2)


@pytest.mark.parametrize("kind", H8.KINDS)
def test_small_batches_beyond_the_capacity_and_in_bad_pages(kind):
    """Of a batch of single tokens and of pairs, only those with a place are written; all is reported."""
    import torch
    for T in (1, 2):
        c = H8.Case(kind, 8, 8, 128, [20 + s for s in range(40)], page=16, D=512, seed=T, max_len=64)
        before, sc = c.kv.clone(), c.sc.clone()
        x = torch.ones(40, T, 512, dtype=torch.bfloat16, device="cuda")
        c.workspace(T)
        c.sl.copy_(torch.tensor([49] * 36 + [65, -3, 0, 40], dtype=torch.int32))
        c.table[:, 3] = 10 ** 6
        c.table[:, 2] = -1
        c.table[0] = torch.arange(4, dtype=torch.int32, device="cuda") + 3
        owned = [3 + 3] if T == 1 else [3 + 2, 3 + 3]
        c.L.lorc_append8(c.ctx, 0, c.cache(), x, T)
        assert c.L.lorc_last_path(c.ctx) == 2 and c.status() == c.L.LORC_ERR_CAPACITY
        changed = (c.kv != before).any(-1)
        rows = {(p, r) for _, p, r in changed.nonzero().tolist()}
        # position 48 (T = 1), 47 and 48 (T = 2), of sequence 0
        want = {(6, 0)} if T == 1 else {(5, 15), (6, 0)}
        assert want <= rows
        assert all(p in owned for p, _ in rows)          # (earlier tokens of the block may be under a larger scale)
        scales = {p for _, p, b, _ in (c.sc != sc).nonzero().tolist()}
        assert scales <= set(owned)
        c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
def test_numbers_that_are_not_finite(kind):
    """They are reported and contained: NaN becomes 0, an infinity the largest code, other heads and blocks are as ever."""
    import torch
    c = H8.Case(kind, 4, 2, 64, [40], D=256, style=H.ROPE_NONE, seed=9)
    w = np.asarray(c.w[1]).copy()
    w[7, 3], w[7, 5] = np.inf, np.nan
    c.L.lorc_load_factors(c.ctx, 0, c.L.LORC_MODE_FULL, 0, 0, H.dev_bf16(c.w[0]), None, H.dev_bf16(w), None)
    x = torch.zeros(1, 2, 256, dtype=torch.bfloat16, device="cuda")
    x[0, 0, 7] = x[0, 1, 7] = 1.0
    # 0 x inf is NaN in every row that meets them; rows of the other weights are finite
    c.workspace(2)
    c.L.lorc_append8(c.ctx, 0, c.cache(), x, 2)
    assert c.status() == c.L.LORC_ERR_ARG
    got = H8.host_codes(c.kv, kind)
    top = C8.LARGEST[kind]
    assert (got[1, 0, 38:40, 3] == top).all() and (got[1, 0, 38:40, 5] == 0).all()
    assert np.isfinite(got).all() and bool(torch.isfinite(c.sc).all())
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("T,lens", [(1, [17, 40]), (2, [40]), (100, [140])])
def test_finite_numbers_beside_others_count_for_the_scale(kind, T, lens, path=None):
    """The largest finite numbers of a block stand next to a NaN and an infinity: codes and scales are the oracle's."""
    c = H8.Case(kind, 8, 8, 128, lens, D=512, style=H.ROPE_NONE, seed=T + 30)
    w = np.asarray(c.w[1]).copy()
    w[:, :16] = w[:, :16] * 16
    bad = w.copy()
    bad[7, 3], bad[7, 5] = np.inf, np.nan
    c.L.lorc_load_factors(c.ctx, 0, c.L.LORC_MODE_FULL, 0, 0, H.dev_bf16(c.w[0]), None, H.dev_bf16(bad), None)
    c.w[1] = w
    at, _ = _exact_x(c, T)
    at[:, -1] = 7
    x = np.zeros((c.b, T, c.D))
    x[np.arange(c.b)[:, None], np.arange(T), at] = 1.0
    want_codes, want_scales = c.codes.copy(), c.scales.copy()
    for s, n in enumerate(c.lens):
        page, row = c.rows_of(s, -(-n // 16) * 16)
        for i in range(2):
            new = np.asarray(c.w[i], dtype=np.float64)[at[s]]
            if i == 1:
                new[:, [3, 5]] = 0.0
            codes = want_codes[i][page, row].reshape(-1, c.H_kv, c.d_h)
            scales = want_scales[i][page[::16], row[::16] // 16]
            C8.write(codes, scales, new.reshape(T, c.H_kv, c.d_h), n, kind)
            want_codes[i][page, row] = codes.reshape(-1, c.n)
            want_scales[i][page[::16], row[::16] // 16] = scales
            if i == 1:
                want_codes[1][s, n - T:n, 3] = np.where(at[s] == 7, C8.LARGEST[kind], 0.0)     # (0 x inf is NaN)
    c.workspace(T)
    c.L.lorc_append8(c.ctx, 0, c.cache(), H.dev_bf16(x), T)
    assert c.status() == c.L.LORC_ERR_ARG
    assert c.L.lorc_last_path(c.ctx) == (path or (2 if T == 100 else 3))
    assert np.array_equal(c.sc.double().cpu().numpy(), want_scales)
    assert np.array_equal(H8.host_codes(c.kv, kind), want_codes)
    c.close()


def test_write_beyond_the_capacity_and_into_bad_pages():
    import torch
    c = H8.Case("int8", 4, 2, 64, [20, 30, 40, 1], page=16, D=256, seed=10, max_len=48)
    before, sc = c.kv.clone(), c.sc.clone()
    x = torch.ones(4, 2, 256, dtype=torch.bfloat16, device="cuda")
    c.workspace(2)
    c.sl.copy_(torch.tensor([49, -3, 40, 1], dtype=torch.int32))
    c.table[2, 2] = 10 ** 6
    c.L.lorc_append8(c.ctx, 0, c.cache(), x, 2)
    assert c.status() == c.L.LORC_ERR_CAPACITY
    # sequence 3 has one token only: its second new token is written, nothing else changes
    page = int(c.table[3, 0])
    changed = (c.kv != before).any(-1)
    assert bool(changed[:, page, 0].all())
    changed[:, page, 0] = False
    assert not bool(changed.any())
    sc[:, page, 0] = c.sc[:, page, 0]
    assert torch.equal(sc, c.sc)
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("heads", [(32, 8, 128), (4, 2, 64)])
def test_a_prompt_and_steps_together(kind, heads):
    """As a program uses them: a prompt in two chunks, then steps, write and attention each time; the attention is that of the
    numbers that the cache holds then, and these stay within their steps of the fp64 keys and values."""
    import torch
    D = 256
    c = H8.Case(kind, *heads, [60, 60], page=16, D=D, seed=11, max_len=80)
    x = H.synth.to_bf16_exact(c.rng.standard_normal((2, 70, D)))
    xd = H.dev_bf16(x)
    done = 0
    for T in (33, 27, 1, 1, 1, 1, 1):
        done += T
        c.lens = [done, done]
        c.sl.fill_(done)
        c.workspace(T)
        cache = c.cache()
        c.L.lorc_append8(c.ctx, 0, cache, xd[:, done - T:done].contiguous(), T)
        q, qd = c.queries(T, scale=1.0)
        out = torch.zeros(2, T, c.H_q, c.d_h, dtype=torch.bfloat16, device="cuda")
        if T == 1:
            c.L.lorc_decode_attn8(c.ctx, 0, cache, qd, out)
        else:
            c.L.lorc_prefill_attn8(c.ctx, 0, cache, qd, out, T)
        c.codes, c.scales = H8.host_codes(c.kv, kind), c.sc.double().cpu().numpy()
        H8.assert_attention(H.host_f64(out), *c.want(q, T), fp16=T > 1 and heads[2] == 128)
    assert c.status() == 0
    for s in range(2):
        for i in range(2):
            new = (x[s, :done].astype(np.float64) @ np.asarray(c.w[i], dtype=np.float64)).reshape(done, c.H_kv, c.d_h)
            if i == 0:
                new = np.stack([c.rotate(new[t], t) for t in range(done)])
            got = c.held(i, s, done)
            page, row = c.rows_of(s, done)
            scale = c.scales[i][page, row // 16][..., None]
            # int8: half a step when written, half a step of the new scale for each time that it doubled: less than one step of the
            # final scale in all.  e4m3: exact but for subnormals
            half = scale if kind == "int8" else 2.0 ** -4 * np.abs(new) + scale * 2.0 ** -9
            assert (np.abs(got - new) <= half + 2.0 ** -12).all()
    c.close()


def test_other_streams_and_a_captured_graph():
    import torch
    c = H8.Case("int8", 8, 2, 128, [400, 900], page=64, D=256, seed=12, max_len=960)
    c.workspace(1)
    x = H.dev_bf16(c.rng.standard_normal((2, 1, 256)))
    q, qd = c.queries()
    out = torch.zeros(2, 8, 128, dtype=torch.bfloat16, device="cuda")
    cache = c.cache()

    def step():
        c.L.lorc_append8(c.ctx, 0, cache, x)
        c.L.lorc_decode_attn8(c.ctx, 0, cache, qd, out)

    step()
    torch.cuda.synchronize()
    want, kv = out.clone(), c.kv.clone()
    out.zero_()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for length in ([400, 900], [401, 77]):
        c.sl.copy_(torch.tensor(length, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(out, got)
        if length == [400, 900]:
            assert torch.equal(got, want) and torch.equal(c.kv, kv)
    assert c.status() == 0
    c.close()


def test_refusals():
    import torch
    L = H.lib()
    c = H8.Case("int8", 8, 2, 128, [40], page=16, D=256, seed=13)
    c.workspace(4)
    q = torch.zeros(1, 8, 128, dtype=torch.bfloat16, device="cuda")
    x = torch.zeros(1, 4, 256, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q)

    def refused(code, call, *a, **k):
        with pytest.raises(L.LorcError) as e:
            call(*a, **k)
        assert e.value.code == code, str(e.value)

    for bad in (dict(k=None), dict(v_scale=None), dict(seq_lens=None), dict(batch=0), dict(max_seq_len=0), dict(max_seq_len=81),
                dict(type=2), dict(page_size=8), dict(page_size=0), dict(max_pages_per_seq=1), dict(n_pages=0),
                dict(k=c.kv.data_ptr() + 8), dict(k_scale=c.sc.data_ptr() + 2), dict(page_table=None, seq_stride=40),
                dict(page_table=None, seq_stride=0)):
        refused(L.LORC_ERR_ARG, L.lorc_decode_attn8, c.ctx, 0, c.cache(**bad), q, out)
        refused(L.LORC_ERR_ARG, L.lorc_append8, c.ctx, 0, c.cache(**bad), x, 1)
        refused(L.LORC_ERR_ARG, L.lorc_prefill_attn8, c.ctx, 0, c.cache(**bad), q, out, 1)
    refused(L.LORC_ERR_ARG, L.lorc_decode_attn8, c.ctx, 0, c.cache(), None, out)
    refused(L.LORC_ERR_ARG, L.lorc_decode_attn8, c.ctx, 0, c.cache(), q, None)
    refused(L.LORC_ERR_ARG, L.lorc_decode_attn8, c.ctx, 0, c.cache(), q.data_ptr() + 2, out)
    refused(L.LORC_ERR_LAYER, L.lorc_decode_attn8, c.ctx, 1, c.cache(), q, out)
    for T in (0, -1, 41):
        refused(L.LORC_ERR_ARG, L.lorc_append8, c.ctx, 0, c.cache(), x, T)
        refused(L.LORC_ERR_ARG, L.lorc_prefill_attn8, c.ctx, 0, c.cache(), q, out, T)
    L.lorc_set_workspace(c.ctx, None)
    refused(L.LORC_ERR_WORKSPACE, L.lorc_decode_attn8, c.ctx, 0, c.cache(), q, out)
    refused(L.LORC_ERR_WORKSPACE, L.lorc_append8, c.ctx, 0, c.cache(), x, 4)
    L.lorc_set_workspace(c.ctx, c.ws, 256)
    refused(L.LORC_ERR_WORKSPACE, L.lorc_append8, c.ctx, 0, c.cache(), x, 4)
    assert L.lorc_cache8_workspace_bytes(c.ctx, 0, 40, 1) == 0 and L.lorc_cache8_workspace_bytes(c.ctx, 1, 40, 0) == 0
    # a compressed layer
    ctx = L.lorc_create(2, 256, 8, 2, 128, 10000.0, max_pos=64)
    a, f = torch.zeros(256, 32, dtype=torch.bfloat16, device="cuda"), torch.zeros(32, 256, dtype=torch.bfloat16, device="cuda")
    L.lorc_load_factors(ctx, 0, L.LORC_MODE_LATENT, 32, 32, a, f, a, f)
    L.lorc_set_workspace(ctx, c.ws)
    refused(L.LORC_ERR_UNSUPPORTED, L.lorc_decode_attn8, ctx, 0, c.cache(), q, out)
    refused(L.LORC_ERR_LAYER, L.lorc_decode_attn8, ctx, 1, c.cache(), q, out)
    L.lorc_destroy(ctx)
    assert c.status() == 0
    c.close()
