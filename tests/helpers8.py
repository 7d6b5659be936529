"""Set-up of the tests of the 8-bit cache: a context with one uncompressed layer, caches with known codes and scales, the
fp64 results from `oracle/cache8_oracle.py`."""
from __future__ import annotations

import numpy as np

from oracle import cache8_oracle as C8
from oracle import lorc_oracle as O

import helpers as H

KINDS = ("int8", "e4m3")


def torch_codes(codes, kind):
    """Codes (float64) as the bytes that the cache holds."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(codes))
    return t.to(torch.int8) if kind == "int8" else t.float().to(torch.float8_e4m3fn).view(torch.int8)


def host_codes(t, kind):
    import torch
    t = t.cpu()
    return (t if kind == "int8" else t.view(torch.float8_e4m3fn).float()).double().numpy()


class Case:
    """One uncompressed layer, its cache (contiguous: page = 0), and what it holds in fp64."""

    def __init__(self, kind, H_q, H_kv, d_h, lens, page=0, D=256, style=0, theta=10000.0, seed=0, max_len=None, flags=0,
                 order=None):
        import torch
        self.L = L = H.lib()
        rng = np.random.default_rng([17, seed])
        self.kind, self.H_q, self.H_kv, self.d_h, self.style, self.theta, self.D = kind, H_q, H_kv, d_h, style, theta, D
        self.G, self.n, self.lens = H_q // H_kv, H_kv * d_h, [int(x) for x in lens]
        b, n = len(lens), self.n
        self.b, self.page = b, page
        self.max_len = max_len or max(1, max(self.lens))
        room = -(-self.max_len // 16) * 16
        if page:
            self.per = -(-room // page)
            n_pages = b * self.per + 2
            self.table_h = rng.permutation(n_pages)[: b * self.per].reshape(b, self.per).astype(np.int32)
            rows, ps = n_pages, page
        else:
            rows, ps = b, room + 16
        self.rows_per_page = ps
        self.codes = C8.round_code(rng.standard_normal((2, rows, ps, n)) * (34 if kind == "int8" else 100), kind)
        self.scales = np.ldexp(1.0, rng.integers(-8, -3, (2, rows, ps // 16, H_kv)))
        self.w = [H.synth.to_bf16_exact(rng.standard_normal((D, n)) / np.sqrt(D)) for _ in range(2)]
        self.ctx = L.lorc_create(1, D, H_q, H_kv, d_h, theta, rope_style=style, max_pos=self.max_len + 40, flags=flags)
        L.lorc_load_factors(self.ctx, 0, L.LORC_MODE_FULL, 0, 0, H.dev_bf16(self.w[0]), None, H.dev_bf16(self.w[1]), None)
        self.upload()
        self.sl = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.table = torch.tensor(self.table_h, device="cuda") if page else None
        self.rng = rng
        self.ws = None

    def upload(self):
        import torch
        self.kv = torch_codes(self.codes, self.kind).cuda()
        self.sc = torch.tensor(self.scales, dtype=torch.float32, device="cuda")

    def cache(self, **over):
        type = {"int8": self.L.LORC_CACHE8_INT8, "e4m3": self.L.LORC_CACHE8_E4M3}[self.kind]
        a = dict(k=self.kv[0], v=self.kv[1], k_scale=self.sc[0], v_scale=self.sc[1], seq_lens=self.sl, batch=self.b,
                 max_seq_len=self.max_len, type=type)
        if self.page:
            a.update(page_table=self.table, page_size=self.page, max_pages_per_seq=self.per, n_pages=self.kv.shape[1])
        else:
            a.update(seq_stride=self.rows_per_page)
        a.update(over)
        return self.L.make_cache8(**a)

    def workspace(self, T=1):
        """Exactly as much as the library asks for, and a guard behind it."""
        import torch
        need = self.L.lorc_cache8_workspace_bytes(self.ctx, self.b, self.max_len, T)
        self.ws = torch.full((need + 256,), 0x5a, dtype=torch.uint8, device="cuda")
        self.need = need
        self.L.lorc_set_workspace(self.ctx, self.ws, need)

    def guard_intact(self):
        return bool((self.ws[self.need:] == 0x5a).all())

    def rows_of(self, s, n):
        """(page, row) of the first n tokens of a sequence."""
        pos = np.arange(n)
        if not self.page:
            return np.full(n, s), pos
        return self.table_h[s, pos // self.page], pos % self.page

    def held(self, i, s, n):
        """Numbers [n, H_kv, d_h] of keys (0) or values (1)."""
        page, row = self.rows_of(s, n)
        return (self.codes[i][page, row].reshape(n, self.H_kv, self.d_h) *
                self.scales[i][page, row // 16][..., None])

    def rotate(self, x, pos):
        """x [heads, d_h] at one position."""
        if self.style == H.ROPE_NONE:
            return x
        return O.rope(x, pos, self.theta, self.style)

    def queries(self, T=1, scale=2.0):
        q = H.synth.to_bf16_exact(scale * self.rng.standard_normal((self.b, T, self.H_q, self.d_h)))
        return q.astype(np.float64), H.dev_bf16(q)

    def want(self, q, T=1):
        """Attention in fp64 [b, T, H_q, d_h], and bounds: sum |q k| / sqrt(d), largest |v|, per row."""
        out = np.zeros(q.shape)
        size, vmax = np.zeros(q.shape[:3] + (1,)), np.zeros(q.shape[:3] + (1,))
        for s, n in enumerate(self.lens):
            if n < T or n <= 0:
                continue
            k, v = self.held(0, s, n), self.held(1, s, n)
            for t in range(T):
                m = n - T + t + 1
                qr = self.rotate(q[s, t], m - 1)
                out[s, t], a = C8.attention(k[:m], v[:m], qr, self.G)
                size[s, t, :, 0] = a
                vmax[s, t, :, 0] = np.repeat(np.abs(v[:m]).max(axis=(0, 2)), self.G)
        return out, size, vmax

    def want_some(self, q, T, some):
        """The same for the queries `some` only."""
        shape = (self.b, len(some), self.H_q)
        out, size, vmax = np.zeros(shape + (self.d_h,)), np.zeros(shape + (1,)), np.zeros(shape + (1,))
        for s, n in enumerate(self.lens):
            k, v = self.held(0, s, n), self.held(1, s, n)
            for i, t in enumerate(some):
                m = n - T + t + 1
                out[s, i], a = C8.attention(k[:m], v[:m], self.rotate(q[s, t], m - 1), self.G)
                size[s, i, :, 0] = a
                vmax[s, i, :, 0] = np.repeat(np.abs(v[:m]).max(axis=(0, 2)), self.G)
        return out, size, vmax

    def status(self):
        return self.L.lorc_sync_status(self.ctx)

    def close(self):
        import torch
        torch.cuda.synchronize()
        self.L.lorc_destroy(self.ctx)
        self.ctx = None


def assert_attention(got, want, size, vmax, fp16=False):
    """Element by element: half a step of the bf16 output, 2^-8 |want|, and the arithmetic.  With A = sum |q_i k_i| / sqrt(d):
    a score in fp32 is off by at most 128 sums of 2^-24 A and 2^-22 A for the rotation and the two fp16 parts of the query,
    together less than 2^-16.5 A; a change of every score by at most e moves a softmax average by at most 2 e max|v|
    (up to second order); exponentials, products and sums of at most 2^13 numbers add less than 2^-15 max|v|; probabilities times
    scale are rounded to fp16 in the numerator, half a step each, which moves the average by at most 2^-11 max|v|.  So
    (2^-11 + 2^-15 (1 + A)) max|v|.  fp16 (the tcgen05 kernel rounds rotated queries and probabilities, and the expanded numbers, to fp16,
    half a step is 2^-11): scores are off by 2^-11 A, 2^-10 A max|v| in the average, probabilities add 2 2^-11 max|v|:
    (2^-10 + 2^-15) (1 + A) max|v|."""
    got = np.asarray(got, dtype=np.float64)
    arithmetic = (2.0 ** -10 + 2.0 ** -15) * (1 + size) if fp16 else 2.0 ** -11 + 2.0 ** -15 * (1 + size)
    bound = 2.0 ** -8 * np.abs(want) + arithmetic * vmax
    excess = np.abs(got - want) - bound
    assert np.isfinite(got).all()
    assert excess.max() <= 0, (float(excess.max()), np.unravel_index(excess.argmax(), excess.shape))
