"""The 8-bit cache where numbers, sizes and masks are at their edges."""
import numpy as np
import pytest

import helpers as H
import helpers8 as H8

pytestmark = pytest.mark.gpu


def _attend(c, q, T):
    """q [b, T, H_q, d_h] (bf16-exact) -> [b, T, H_q, d_h]; T = 1 by lorc_decode_attn8."""
    import torch
    qd = H.dev_bf16(q)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    c.workspace(T)
    if T == 1:
        c.L.lorc_decode_attn8(c.ctx, 0, c.cache(), qd, out)
    else:
        c.L.lorc_prefill_attn8(c.ctx, 0, c.cache(), qd, out, T)
    return H.host_f64(out)


def _assert_weights(c, q, got, T, some=None, fp16=False):
    """Every element against the formula, with a bound by the weights that the tokens have.  w_i: the softmax weights, c_i: the scales
    of the values, M: the largest code, B = sum w_i max|v_i|, A = max_i sum |q k_i| / sqrt(d).
      2^-8 |want|                half a step of the output
      2^-15 (1 + A) B            scores, exponentials and sums in fp32 (as in assert_attention)
      2^-11 B                    half a step of a weight w_i c_i as an fp16 number
      N 2^-32 M max w_i c_i      where it is a subnormal one: half a step is 2^-25, and the heaviest weight stands at 2^7 or more
      N 2^-126 max|v|            weights that fp32 does not hold
    fp16 (tcgen05): queries, keys and values are rounded too, 2^-10 (1 + A) B as in assert_attention."""
    M = {"int8": 127.0, "e4m3": 448.0}[c.kind]
    for s, n in enumerate(c.lens):
        page, row = c.rows_of(s, n)
        k, v, cv = c.held(0, s, n), c.held(1, s, n), np.abs(c.scales[1][page, row // 16])
        for t in range(T) if some is None else some:
            m = n - T + t + 1
            qr = c.rotate(q[s, t], m - 1)
            for h in range(c.H_q):
                g = h // c.G
                x = k[:m, g] @ qr[h] / np.sqrt(c.d_h)
                A = (np.abs(k[:m, g]) @ np.abs(qr[h])).max() / np.sqrt(c.d_h)
                w = np.exp(x - x.max())
                w /= w.sum()
                want, most = w @ v[:m, g], np.abs(v[:m, g]).max(-1)
                B = w @ most
                bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -10 * (1 + A) if fp16 else 2.0 ** -11) * B + 2.0 ** -15 * (1 + A) * B + \
                    m * 2.0 ** -32 * M * (w * cv[:m, g]).max() + m * 2.0 ** -126 * most.max()
                off = np.abs(got[s, t, h] - want) - bound
                assert np.isfinite(got[s, t, h]).all() and off.max() <= 0, (s, t, h, float(off.max()), float(np.abs(want).max()))


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("T", [1, 2, 3, 5])
@pytest.mark.parametrize("small", [0.0, 2.0 ** -126, 2.0 ** -100, 2.0 ** -20])
def test_large_scales_beside_small_ones(kind, T, small):
    """The last block of a sequence has far larger values than all others, and most of the queries do not see it (or it has no weight
    that fp32 holds): what they do see counts in full."""
    c = H8.Case(kind, 4, 2, 64, [17, 33, 50], style=2, seed=T)
    M = 127.0 if kind == "int8" else 448.0
    q = H.synth.to_bf16_exact(np.repeat(c.rng.standard_normal((c.b, 1, c.H_kv, c.d_h)), c.G, axis=2)).astype(np.float64)
    q = np.repeat(q, T, axis=1)
    c.scales[0] = 2.0 ** -9 if kind == "int8" else 2.0 ** -11
    for large in (8, 9, 28, 30, 60, 80):
        for low in (False, True):
            for s, n in enumerate(c.lens):
                last = (n - 1) // 16
                c.scales[1][s] = small
                c.scales[1][s, last] = 2.0 ** large
                for h in range(c.H_kv):
                    x = q[s, 0, h * c.G]
                    unit = np.clip(np.rint(-x / np.abs(x).max() * 31), -31, 31)
                    unit = np.where(np.abs(unit) > 16, 2 * np.rint(unit / 2), unit)         # (numbers of both types)
                    # a score of -200: no weight in fp32, and less than 2^-126 of the smallest values' share
                    c.codes[0][s, 16 * last:, h * c.d_h:(h + 1) * c.d_h] = unit if low else unit * 0
                    c.scales[0][s, last, h] = np.float32(200.0 * np.sqrt(c.d_h) / -(unit @ x))
            assert np.abs(c.codes).max() <= M
            c.upload()
            _assert_weights(c, q, _attend(c, q, T), T)
            c.status()
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("T", [1, 3])
def test_queries_of_any_size(kind, T):
    """Queries of 2^120 on keys of 2^-120: the scores are ordinary ones."""
    c = H8.Case(kind, 4, 2, 64, [50, 300], style=0, seed=T + 40)
    q = H.synth.to_bf16_exact(c.rng.standard_normal((c.b, T, c.H_q, c.d_h))).astype(np.float64)
    for up in (90, 100, 116, 120):
        c.scales[0] = 2.0 ** (-up - 6)
        c.upload()
        big = np.ldexp(q, up)
        _assert_weights(c, big, _attend(c, big, T), T)
        assert c.status() == 0
    c.close()


def _sinks(c, every):
    """One token in `every` takes nearly all of the weight and has no value, the others stand 26 powers of two below it with values
    of one sign.  -> the first element of a query"""
    top, rest = 100.0 if c.kind == "int8" else 96.0, 2.0 ** -5
    c.codes[0][:] = 0.0
    c.codes[0][:, ::every, ::c.d_h] = top
    c.scales[0][:] = rest
    c.codes[1] = np.abs(c.codes[1])
    c.codes[1][:, ::every] = 0.0
    c.scales[1][:] = 2.0 ** -4
    c.upload()
    return float(H.synth.to_bf16_exact(np.array([18.2 * np.sqrt(c.d_h) / (top * rest)]))[0])


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("T,heads,lens", [(1, (2, 1, 64), [5000]), (3, (2, 1, 64), [5000]), (1, (8, 1, 128), [100, 20000, 1])])
def test_many_tokens_far_below_the_heaviest(kind, T, heads, lens):
    """(A heavy token for every warp of every block: each has a reference of its own.)"""
    c = H8.Case(kind, *heads, lens, style=2, seed=50)
    q = np.zeros((c.b, T, c.H_q, c.d_h))
    q[..., 0] = _sinks(c, 32)
    _assert_weights(c, q, _attend(c, q, T), T)
    assert c.L.lorc_last_path(c.ctx) == 3 and c.status() == 0
    c.close()


@pytest.mark.parametrize("heads", [(4, 1, 128), (6, 2, 64)])
@pytest.mark.parametrize("T,N", [(400, 20000), (2500, 2500)])
def test_chunks_far_below_the_heaviest(heads, T, N):
    """(A heavy token in every tile of keys: blocks may share them.)"""
    c = H8.Case("int8", *heads, [N], style=2, seed=51)
    q = np.zeros((1, T, c.H_q, c.d_h))
    q[..., 0] = _sinks(c, 128)
    got = _attend(c, q, T)
    assert c.L.lorc_last_path(c.ctx) == 2 and c.status() == 0
    _assert_weights(c, q, got, T, some=(40, T // 2, T - 1), fp16=True)
    c.close()


def test_chunks_of_the_latent_cache_far_below_the_heaviest():
    """The same kernel over reconstructed keys and values: factors of rank 128 that are the identity."""
    import torch
    L = H.lib()
    N, T, d = 20000, 200, 128
    ctx = L.lorc_create(1, 256, 32, 8, d, 10000.0, rope_style=H.ROPE_NONE, max_pos=N)
    eye = torch.eye(d, dtype=torch.bfloat16, device="cuda").repeat(1, 8).contiguous()
    a = torch.zeros(256, d, dtype=torch.bfloat16, device="cuda")
    L.lorc_load_factors(ctx, 0, L.LORC_MODE_LATENT, d, d, a, eye, a, eye)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = torch.zeros(1, N, d, device="cuda"), torch.rand(1, N, d, generator=g, device="cuda")
    k[0, ::128, 0], v[0, ::128] = 3.125, 0.0
    k, v = k.bfloat16(), v.bfloat16()
    sl = torch.tensor([N], dtype=torch.int32, device="cuda")
    cache = L.make_cache(k, v, sl, 1, N, seq_stride=N)
    ws = torch.zeros(L.lorc_prefill_workspace_bytes(ctx, 1, N, T), dtype=torch.uint8, device="cuda")
    L.lorc_set_workspace(ctx, ws)
    q = torch.zeros(1, T, 32, d, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 18.2 * np.sqrt(d) / 3.125
    out = torch.zeros_like(q)
    L.lorc_prefill_attn(ctx, 0, cache, q, out, T)
    assert L.lorc_sync_status(ctx) == 0 and L.lorc_last_path(ctx) == 2
    x = (float(q[0, 0, 0, 0]) * k[0, :, 0].double()) / np.sqrt(d)
    for t in (0, 77, T - 1):
        m = N - T + t + 1
        w = torch.softmax(x[:m], 0)
        want = (w @ v[0, :m].double()).cpu().numpy()
        # (as _assert_weights, fp16: A = 18.2, the values do not exceed 1)
        B = float(w @ v[0, :m].double().abs().amax(-1))
        bound = 2.0 ** -8 * want + (2.0 ** -10 + 2.0 ** -15) * 19.2 * B + m * 2.0 ** -32 * float(w.max())
        assert (np.abs(H.host_f64(out[0, t]) - want) <= bound).all(), t
    L.lorc_destroy(ctx)


# (8 KV heads in groups of 1, 4, 6: 128-wide blocks with and without rows that are nobody's; 64-wide ones; what `way` says is by the
# rules for 148 SMs: streamed, keys shared by all units, by none, by those of the last round)
MASKS = [((4, 2, 64), 1, [3000, 70], 0), ((32, 8, 128), 1, [2100, 17], 64), ((8, 2, 128), 5, [4000, 5, 130], 16),
         ((4, 2, 64), 33, [2500, 33], 48), ((32, 8, 128), 150, [5000], 64), ((32, 8, 128), 700, [700], 0),
         ((64, 8, 128), 300, [300, 4000], 128), ((6, 2, 128), 150, [5000], 0), ((10, 2, 128), 1500, [1500] * 4, 64),
         ((7, 1, 128), 1500, [1500] * 4, 0), ((32, 8, 64), 150, [5000], 16), ((32, 8, 64), 700, [700], 64),
         ((64, 8, 64), 300, [300, 4000], 0)]


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("heads,T,lens,page", MASKS)
def test_masks_to_the_token(kind, heads, T, lens, page):
    """Keys are zero, so every token that a query sees has the same weight; from the chunk on a token has one number that is not
    zero, also behind the sequence's end.  A result is a count divided by a length: half a step of the output, and some sums
    in fp32."""
    c = H8.Case(kind, *heads, lens, page=page, style=2, seed=70)
    c.codes[:] = 0.0
    c.scales[:] = 2.0 ** -3
    want = np.zeros((c.b, T, heads[2]))
    for s, n in enumerate(c.lens):
        room = -(-n // 16) * 16
        pg, row = c.rows_of(s, room)
        for pos in range(n - T, room):
            at = pos % c.d_h
            c.codes[1][pg[pos], row[pos], at::c.d_h] = 64.0
            if pos < n:
                want[s, pos - (n - T):, at] += 8.0
        want[s] /= np.arange(n - T, n)[:, None] + 1
    c.upload()
    q = H.synth.to_bf16_exact(c.rng.standard_normal((c.b, T, c.H_q, c.d_h))).astype(np.float64)
    got = _attend(c, q, T)
    off = np.abs(got - want[:, :, None]) - (2.0 ** -8 + 2.0 ** -15) * want[:, :, None]
    assert off.max() <= 0, np.unravel_index(off.argmax(), off.shape)
    assert c.L.lorc_last_path(c.ctx) == (2 if T > 100 else 3)
    assert c.status() == 0 and c.guard_intact()
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("heads,T,lens,page", [m for m in MASKS if m[1] > 100])
def test_chunks_on_the_tensor_cores(kind, style, heads, T, lens, page):
    """Every form of the tcgen05 kernel (all units whole, all shared, those of the last round shared; heads of 128 in groups that fill
    a block or not, interleaved, heads of 64), and that it is the one that runs."""
    c = H8.Case(kind, *heads, lens, page=page, style=style, theta=500000.0, seed=71)
    q = H.synth.to_bf16_exact(c.rng.standard_normal((c.b, T, c.H_q, c.d_h))).astype(np.float64)
    got = _attend(c, q, T)
    assert c.L.lorc_last_path(c.ctx) == 2 and c.status() == 0 and c.guard_intact()
    some = np.unique(np.r_[0, 1, T // 2, T - 1, c.rng.integers(0, T, 4)])
    H8.assert_attention(got[:, some], *c.want_some(q, T, some), fp16=True)
    c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("b,T,D,path", [(2, 1, 256, 3), (40, 1, 512, 2), (9, 5, 512, 2), (2, 100, 512, 2), (1, 3, 200, 3)])
def test_a_write_beside_tokens_under_any_scale(kind, b, T, D, path):
    """Earlier tokens of a block may stand under a scale of either sign: the larger one in magnitude stays, and the numbers that they
    stand for stay what they are."""
    import torch
    from oracle import cache8_oracle as C8
    lens = [T + 1 + (29 * s) % 67 for s in range(b)]
    c = H8.Case(kind, 8, 8, 128, lens, D=D, style=H.ROPE_NONE, seed=T + b)
    c.scales *= np.where(c.rng.random(c.scales.shape) < 0.5, -1.0, 1.0) * np.ldexp(1.0, c.rng.integers(-4, 5, c.scales.shape))
    c.upload()
    at = c.rng.integers(0, D, (b, T))
    x = np.zeros((b, T, D))
    x[np.arange(b)[:, None], np.arange(T), at] = 1.0
    want_codes, want_scales = c.codes.copy(), c.scales.copy()
    for s, n in enumerate(c.lens):
        for i in range(2):
            new = np.asarray(c.w[i], dtype=np.float64)[at[s]].reshape(T, c.H_kv, c.d_h)
            codes, scales = want_codes[i][s].reshape(-1, c.H_kv, c.d_h), want_scales[i][s]
            for b0 in range((n - T) // 16 * 16, n, 16):
                start, end = max(b0, n - T), min(b0 + 16, n)
                fresh = new[start - (n - T):end - (n - T)]
                scale, before = C8.scale_for(np.abs(fresh).max(axis=(0, 2)), kind), scales[b0 // 16]
                if start > b0:
                    scale = np.where(np.abs(before) > scale, before, scale)
                    codes[b0:start] = C8.round_code(codes[b0:start] * (before / scale)[None, :, None], kind)
                codes[start:end] = C8.round_code(fresh / scale[None, :, None], kind)
                scales[b0 // 16] = scale
    c.workspace(T)
    c.L.lorc_append8(c.ctx, 0, c.cache(), H.dev_bf16(x), T)
    assert c.L.lorc_last_path(c.ctx) == path
    assert np.array_equal(c.sc.double().cpu().numpy(), want_scales)
    assert np.array_equal(H8.host_codes(c.kv, kind), want_codes)
    assert c.status() == 0
    c.close()


def test_many_new_tokens_under_a_long_cache():
    """64 sequences, 8192 new tokens each, in a cache that may hold 131072 of each: write and attention are those of a shorter bound."""
    import torch
    L = H.lib()
    b, T, D, d, room, most = 64, 8192, 64, 64, 131072, 8704
    g = torch.Generator(device="cuda").manual_seed(1)
    ctx = L.lorc_create(1, D, 1, 1, d, 10000.0, rope_style=0, max_pos=room)
    w = torch.randn(2, D, d, generator=g, device="cuda").mul_(D ** -0.5).bfloat16()
    L.lorc_load_factors(ctx, 0, L.LORC_MODE_FULL, 0, 0, w[0], None, w[1], None)
    lens = T + torch.randint(0, most - T, (b,), generator=g, device="cuda", dtype=torch.int32)
    x = torch.randn(b, T, D, generator=g, device="cuda").bfloat16()
    q = torch.randn(b, T, 1, d, generator=g, device="cuda").bfloat16()
    held = []
    for bound in (most, room):
        kv = torch.zeros(2, b, room, d, dtype=torch.int8, device="cuda")
        sc = torch.full((2, b, room // 16, 1), 2.0 ** -100, device="cuda")
        cache = L.make_cache8(kv[0], kv[1], sc[0], sc[1], lens, b, bound, L.LORC_CACHE8_INT8, seq_stride=room)
        need = L.lorc_cache8_workspace_bytes(ctx, b, bound, T)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        L.lorc_set_workspace(ctx, ws)
        L.lorc_append8(ctx, 0, cache, x, T)
        out = torch.zeros_like(q)
        L.lorc_prefill_attn8(ctx, 0, cache, q, out, T)
        assert L.lorc_sync_status(ctx) == 0
        held.append((kv, sc, out))
    assert torch.equal(held[0][0], held[1][0]) and torch.equal(held[0][1], held[1][1])
    # the same averages of probabilities that were rounded to fp16 (2 2^-11 max|v| each way), rounded once each
    kv, sc, out = held[1]
    most = 127 * float(sc.max())
    assert bool(((out.float() - held[0][2].float()).abs() <= 2.0 ** -7 * out.float().abs() + 2.0 ** -9 * most).all())
    inv = 10000.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
    for s, t in ((0, 0), (17, 4000), (63, T - 1)):
        m = int(lens[s]) - T + t + 1
        k, v = [kv[i, s, :m].double() * sc[i, s].double().repeat_interleave(16, 0)[:m] for i in range(2)]
        cs, sn = torch.cos((m - 1) * inv), torch.sin((m - 1) * inv)
        a, z = q[s, t, 0].double().chunk(2)
        qr = torch.cat([a * cs - z * sn, a * sn + z * cs])
        want, size = torch.softmax(k @ qr / d ** 0.5, 0) @ v, float((k.abs() @ qr.abs()).max()) / d ** 0.5
        H8.assert_attention(out[s, t].double().cpu().numpy(), want.cpu().numpy(), size, float(v.abs().max()), fp16=True)
    L.lorc_destroy(ctx)


def test_sizes_that_are_refused():
    """2^30 tokens in a call, and lists of 2^30 units of 64 tokens for the streaming kernel; nothing of the memory is touched."""
    import torch
    L = H.lib()
    ctx = L.lorc_create(1, 64, 1, 1, 64, 10000.0, max_pos=65536)
    w = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    L.lorc_load_factors(ctx, 0, L.LORC_MODE_FULL, 0, 0, w, None, w, None)
    some = torch.zeros(4096, dtype=torch.int32, device="cuda")
    for batch, T, calls in ((1 << 14, 65536, "wp"), (1 << 20, 1, "d"), (1 << 20, 1024, "wp")):
        cache = L.make_cache8(some, some, some, some, some, batch, 65536, L.LORC_CACHE8_INT8, seq_stride=65536)
        for c, call in (("w", lambda: L.lorc_append8(ctx, 0, cache, some, T)), ("d", lambda: L.lorc_decode_attn8(ctx, 0, cache, some, some)),
                        ("p", lambda: L.lorc_prefill_attn8(ctx, 0, cache, some, some, T))):
            if c in calls:
                with pytest.raises(L.LorcError) as e:
                    call()
                assert e.value.code == L.LORC_ERR_ARG, str(e.value)
    assert L.lorc_sync_status(ctx) == 0
    L.lorc_destroy(ctx)


def _step(c, T):
    """Buffers and calls of a step: a chunk of T tokens is written and attended to, then its last token as a step of its own."""
    import torch
    x = H.dev_bf16(c.rng.standard_normal((c.b, T, c.D)))
    last = x[:, -1:].contiguous()
    q, qd = c.queries(T, scale=1.0)
    q1 = qd[:, -1].contiguous()
    out, dec = torch.zeros_like(qd), torch.zeros_like(q1)
    cache = c.cache()
    c.workspace(T)

    def calls():
        c.L.lorc_append8(c.ctx, 0, cache, x, T)
        c.L.lorc_prefill_attn8(c.ctx, 0, cache, qd, out, T)
        c.path = c.L.lorc_last_path(c.ctx)
        c.L.lorc_append8(c.ctx, 0, cache, last, 1)
        c.L.lorc_decode_attn8(c.ctx, 0, cache, q1, dec)

    return calls, [out, dec, c.kv, c.sc]


@pytest.mark.parametrize("kind", H8.KINDS)
@pytest.mark.parametrize("T,path", [(3, 3), (150, 2), (700, 2)])
def test_a_captured_chunk_under_other_lengths(kind, T, path):
    """One graph, replayed with other lengths (empty, shorter than the chunk, the longest): what the calls give."""
    import torch
    c = H8.Case(kind, 32, 8, 128, [T, T + 900, T + 40], page=64, D=512, seed=80, max_len=T + 1000)
    calls, held = _step(c, T)
    calls()
    assert c.path == path and c.status() == 0
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls()
    for lens in ([T, T + 900, T + 40], [T + 17, T + 1000, T], [0, T + 1, T - 1], [T + 500, T + 499, T + 498]):
        c.sl.copy_(torch.tensor(lens, dtype=torch.int32))
        kv, sc = c.kv.clone(), c.sc.clone()
        graph.replay()
        torch.cuda.synchronize()
        got, status = [t.clone() for t in held], c.status()
        c.kv.copy_(kv)
        c.sc.copy_(sc)
        for t in held[:2]:
            t.fill_(7.0)
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, held)), lens
        assert status == c.status() or min(lens) < T        # (of several errors one is kept)
    assert c.guard_intact()
    c.close()


def test_two_contexts_at_once():
    """Contexts share nothing: on two streams at the same time they give what they give alone."""
    import torch
    cases = [(H8.Case("int8", 32, 8, 128, [150 + 37 * s for s in range(6)], page=64, D=512, seed=81, max_len=600), 150),
             (H8.Case("e4m3", 12, 6, 64, [40 + s % 90 for s in range(40)], D=1024, seed=82, max_len=200), 5)]
    steps = [_step(c, T) for c, T in cases]
    alone = []
    for calls, held in steps:
        calls()
        torch.cuda.synchronize()
        alone.append([t.clone() for t in held])
    streams = [torch.cuda.Stream() for _ in cases]
    graphs = []
    for (calls, _), stream in zip(steps, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            for _ in range(4):
                calls()
        graphs.append(graph)
    for _ in range(25):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for (_, held), want, (c, _) in zip(steps, alone, cases):
        assert all(torch.equal(a, b) for a, b in zip(held, want))
        assert c.status() == 0 and c.guard_intact()
        c.close()


@pytest.mark.parametrize("kind", H8.KINDS)
def test_chunks_whose_pages_lie_outside_the_pool(kind):
    """Expanded chunks: such tokens count as zeros (status CAPACITY), the other sequences are as ever."""
    import torch
    c = H8.Case(kind, 32, 8, 128, [1500, 400], page=32, seed=83)
    c.table[0, 2], c.table[0, 40] = -1, 10 ** 6
    q = H.synth.to_bf16_exact(c.rng.standard_normal((c.b, 200, c.H_q, c.d_h))).astype(np.float64)
    got = _attend(c, q, 200)
    assert c.L.lorc_last_path(c.ctx) == 2 and c.status() == c.L.LORC_ERR_CAPACITY and c.guard_intact()
    for page in (c.table_h[0, 2], c.table_h[0, 40]):
        c.codes[:, page] = 0.0
    some = np.array([0, 63, 199])
    H8.assert_attention(got[:, some], *c.want_some(q, 200, some), fp16=True)
    c.close()


@pytest.mark.parametrize("b", [5, 16])
def test_sums_of_a_few_tokens(b):
    """Products of one sign, so that what the tensor cores' fp32 sums lose adds up: every code is the fp64 projection's, unless that lies
    within 2^-20 of the products' sum of a border between two.  Each of 8 MMAs in a row (128 products) loses an ulp, 2^-23, of
    their sum so far: 2^-21; eight such pieces per warp are added up in fp32, 2^-22, and those of eight warps, 3 2^-24: together
    less than 2^-20."""
    import torch
    D = 8192
    for seed in range(3):
        c = H8.Case("int8", 8, 8, 128, [16] * b, D=D, style=H.ROPE_NONE, seed=seed)
        w = [H.synth.to_bf16_exact(np.abs(c.rng.standard_normal((D, c.n))) / np.sqrt(D)) for _ in range(2)]
        c.L.lorc_load_factors(c.ctx, 0, c.L.LORC_MODE_FULL, 0, 0, H.dev_bf16(w[0]), None, H.dev_bf16(w[1]), None)
        x = H.dev_bf16(H.synth.to_bf16_exact(np.abs(c.rng.standard_normal((b, 1, D)))))
        c.sc.fill_(2.0 ** -100)
        c.workspace(1)
        c.L.lorc_append8(c.ctx, 0, c.cache(), x, 1)
        assert c.L.lorc_last_path(c.ctx) == 3 and c.status() == 0
        for i in range(2):
            new = (x[:, 0].double() @ H.dev_bf16(w[i]).double()).view(b, 8, 128)
            scale = c.sc[i, :, 0].double()[..., None]
            got = c.kv[i, :, 15].double().view(b, 8, 128)
            near = (new / scale - (torch.floor(new / scale) + 0.5)).abs() * scale <= 2.0 ** -20 * new
            assert bool(((got == torch.round(new / scale)) | near).all())
        c.close()
