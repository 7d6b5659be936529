"""The operators of the 8-bit key/value cache and of the pages that caches live in, as they are measured.

The cache of an uncompressed layer in 8 bits: codes (int8, or e4m3 floating point) with one fp32 scale for every block of 16
tokens and KV head; a cached number is code x scale.

  write    lorc_append8: keys and values of T new tokens per sequence are projected, keys rotated, both quantised.  The scale
           of a block is the smallest power of two with which its new numbers do not exceed the largest code (127, or 448),
           and not less than the scale of the rows that the block holds already; these are re-expressed where it grows.
  decode   lorc_decode_attn8: attention of one query per sequence and head over the cached tokens
  chunk    lorc_prefill_attn8: attention of the T newest tokens of every sequence, causal among themselves
  fork     lorc_pages_free, lorc_pages_fork, lorc_pages_grow: a step of a search over several continuations.  The previous
           children give their pages back, new ones share the full pages of their parents and take a copy of the last,
           partly filled one, and get room for a token.  Pages that are needed are the lowest free ones, in the order of the list.
  compact  lorc_pages_compact: the used pages behind the first n_used move into the free ones before it, both in ascending
           order, and the page tables follow

Keys of an attention case: D, heads, kv_heads, d_head, theta (model geometry), type ("int8", "e4m3"), rope ("half",
"interleaved", "none"), batch, len_min, len_max (cached tokens per sequence, new ones included), T (new tokens per sequence),
page (tokens per page in random page order; 0: contiguous), q_scale (standard deviation of the query elements).
Keys of a page case: layers, pages, page, width (numbers per token, in each of a layer's two caches), form ("bf16", or "int8"
with scales), and parents, children (of each parent), len_min, len_max; or rows, len_min, len_max, keep (share of the rows
that still live).
"""
import math
from types import SimpleNamespace

import torch

own = False

BLOCK = 16                                   # tokens that share a scale
LARGEST = {"int8": 127.0, "e4m3": 448.0}
CODE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
GEOMETRY = {
    "8b": dict(D=4096, heads=32, kv_heads=8, d_head=128, theta=500000.0),
    "70b": dict(D=8192, heads=64, kv_heads=8, d_head=128, theta=500000.0),
    "tiny": dict(D=256, heads=4, kv_heads=2, d_head=64, theta=10000.0),
}


def _attention(op, geometry, type, batch, len_min, len_max, T=1, page=0, rope="half", q_scale=4.0):
    return dict(GEOMETRY[geometry], op=op, type=type, batch=batch, len_min=len_min, len_max=len_max, T=T, page=page, rope=rope,
                q_scale=q_scale)


def _fork(layers, pages, page, width, form, parents, children, len_min, len_max):
    return dict(op="fork", layers=layers, pages=pages, page=page, width=width, form=form, parents=parents, children=children,
                len_min=len_min, len_max=len_max)


def _compact(layers, page, width, form, rows, len_min, len_max, keep):
    # pages: what the rows take at their longest
    return dict(op="compact", layers=layers, pages=rows * -(-len_max // page), page=page, width=width, form=form, rows=rows,
                len_min=len_min, len_max=len_max, keep=keep)


def listed():
    c = {}
    # the smallest attention call: one short sequence, 64-wide heads; launches and latency only
    c["decode_tiny"] = _attention("decode", "tiny", "e4m3", 1, 129, 129)
    # the batch that the uncompressed mode is measured with
    c["decode_batch"] = _attention("decode", "8b", "int8", 16, 4129, 4129)
    # few long sequences
    c["decode_long"] = _attention("decode", "8b", "e4m3", 4, 32777, 32777)
    # a ragged serving batch over a paged cache, eight query heads per KV head
    c["decode_ragged"] = _attention("decode", "70b", "int8", 64, 512, 16384, page=64)
    # a decode step's cache write: one token for each of 16 sequences (the cache is short: the write does not see its length)
    c["write_step"] = _attention("write", "8b", "int8", 16, 20, 90)
    # the cache write of prompt chunks, paged, odd lengths
    c["write_chunk"] = _attention("write", "8b", "e4m3", 4, 777, 1003, T=777, page=64)
    # a whole prompt of one user
    c["chunk_prompt"] = _attention("chunk", "8b", "e4m3", 1, 777, 777, T=777)
    # chunked prompt processing of a batch over a paged cache
    c["chunk_batch"] = _attention("chunk", "8b", "int8", 8, 4096, 4096, T=512, page=64)
    # four continuations of one short sequence, one small layer: latency
    c["fork_tiny"] = _fork(1, 32, 16, 32, "bf16", 1, 4, 129, 129)
    # eight continuations for each of eight sequences over eight layers of latents
    c["fork_batch"] = _fork(8, 1024, 64, 384, "bf16", 8, 8, 2000, 4129)
    # a small pool after a few sequences have ended
    c["compact_small"] = _compact(1, 16, 256, "int8", 16, 20, 256, 0.5)
    # a serving pool of 8-bit caches over eight layers after half of the sequences have ended
    c["compact_pool"] = _compact(8, 64, 1024, "int8", 32, 512, 2048, 0.5)
    return [dict(v, name=k) for k, v in c.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = [max(work(c)[k] for c in listed()) for k in ("bytes", "flops")]
    while True:
        c = _draw(rng)
        w = work(c)
        if w["bytes"] <= most[0] and w["flops"] <= most[1]:
            return c


def _draw(rng):
    what = rng.choice(["tiny", "single", "batch", "batch", "long", "ragged", "write", "write", "chunk", "chunk", "fork", "compact"])
    geometry = rng.choice(["8b", "8b", "70b", "tiny"])
    more = dict(type=rng.choice(["int8", "e4m3"]), page=rng.choice([0, 0, 16, 32, 64, 128]), q_scale=rng.choice([1.0, 4.0, 16.0]),
                rope=rng.choice(["half", "half", "half", "interleaved", "none"]))
    if what in ("tiny", "single"):
        n = _log_int(rng, 1, 8000)
        return _attention("decode", "tiny" if what == "tiny" else geometry, batch=rng.randint(1, 4), len_min=max(1, n // 2), len_max=n, **more)
    if what == "batch":
        n = _log_int(rng, 200, 8200)
        return _attention("decode", geometry, batch=rng.randint(3, 48), len_min=max(1, n // rng.choice([1, 8])), len_max=n, **more)
    if what == "long":
        n = _log_int(rng, 16000, 131000)
        return _attention("decode", geometry, batch=rng.randint(1, 4), len_min=n, len_max=n, **more)
    if what == "ragged":
        n = _log_int(rng, 1000, 16384)
        return _attention("decode", geometry, batch=rng.randint(8, 64), len_min=max(1, n // 32), len_max=n, **dict(more, page=rng.choice([16, 32, 64, 128])))
    if what == "write":
        T = _log_int(rng, 1, 1100)
        b = max(1, min(rng.randint(1, 24), 4400 // T))
        return _attention("write", geometry, batch=b, len_min=T, len_max=T + rng.randint(0, 300), T=T, **more)
    if what == "chunk":
        T, b = _log_int(rng, 2, 1100), rng.randint(1, 8)
        return _attention("chunk", geometry, batch=b, len_min=T, len_max=T + rng.choice([0, _log_int(rng, 1, 4000)]), T=T, **more)
    page, width = rng.choice([16, 32, 64, 128]), 8 * rng.randint(4, 128)
    if what == "fork":
        p, k, n = rng.randint(1, 8), rng.randint(1, 8), _log_int(rng, 10, 4200)
        need = p * (n // page + 2) + 3 * p * k
        return _fork(rng.randint(1, 8), need + rng.randint(0, 300), page, width, "bf16", p, k, max(1, n // 3), n)
    width = rng.choice([128, 256, 512, 1024])
    return _compact(rng.randint(1, 8), page, width, rng.choice(["bf16", "int8"]), rng.randint(4, 32), 10, _log_int(rng, 40, 2100),
                    rng.uniform(0.1, 0.9))


# ---- inputs ----------------------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _cache(case, seed):
    """Lengths, page table, codes kv [2, pages, page, n] and scales [2, pages, page / 16, kv_heads]; a contiguous cache is one
    page per sequence in order.  Keys and values are Gaussian; the scales are powers of two, as the write leaves them."""
    g = _generator(seed)
    b, T, ps, n = case["batch"], case["T"], case["page"], case["kv_heads"] * case["d_head"]
    room = -(-(case["len_max"] + 2 * BLOCK) // BLOCK) * BLOCK
    i = SimpleNamespace(g=g, lens=torch.randint(max(T, case["len_min"]), case["len_max"] + 1, (b,), generator=g, device="cuda", dtype=torch.int32))
    if ps:
        per = -(-room // ps)
        i.table = torch.randperm(b * per, generator=g, device="cuda").to(torch.int32).view(b, per)
        pages = b * per
    else:
        i.table, pages, ps = None, b, room
    i.rows_per_page = ps
    noise = torch.randn(2, pages, ps, n, generator=g, device="cuda", dtype=torch.bfloat16)
    if case["type"] == "int8":
        i.kv = noise.mul_(34.0).round_().clamp_(-127, 127).to(torch.int8)
    else:
        i.kv = noise.mul_(90.0).clamp_(-448, 448).to(torch.float8_e4m3fn)
    step = torch.randint(-6, -4, (2, pages, ps // BLOCK, case["kv_heads"]), generator=g, device="cuda")
    i.scale = torch.exp2(step.float() - (0 if case["type"] == "int8" else 1))
    return i


def _pool(case, g, pages):
    if case["form"] == "bf16":
        return torch.randn(case["layers"], 2, pages, case["page"], case["width"], generator=g, device="cuda", dtype=torch.bfloat16), None
    codes = torch.randint(-127, 128, (case["layers"], 2, pages, case["page"], case["width"]), generator=g, device="cuda", dtype=torch.int8)
    heads = case["width"] // 128
    step = torch.randint(-8, -4, (case["layers"], 2, pages, case["page"] // BLOCK, heads), generator=g, device="cuda")
    return codes, torch.exp2(step.float())


def _tables(case, seed):
    """A pool in the middle of its life: page tables, lengths, and how many rows hold each page (0: free)."""
    g = _generator(seed)
    ps, pages = case["page"], case["pages"]
    i = SimpleNamespace(page=ps)
    lens_of = lambda k: torch.randint(case["len_min"], case["len_max"] + 1, (k,), generator=g, device="cuda", dtype=torch.int32)  # noqa: E731
    if case["op"] == "fork":
        p, k = case["parents"], case["children"]
        rows, per = p + p * k, case["len_max"] // ps + 2
        lens = torch.cat([lens_of(p), torch.ones(p * k, device="cuda", dtype=torch.int32)])
    else:
        rows, per = case["rows"], -(-case["len_max"] // ps)
        lens = lens_of(rows)
        gone = torch.randperm(rows, generator=g, device="cuda")[: rows - max(1, int(rows * case["keep"]))]
        lens[gone] = 0
    # the rows' pages lie anywhere in the pool
    held = -(-lens // ps)
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    place = torch.cumsum(held, 0) - held
    col = torch.arange(per, device="cuda")
    live = col < held[:, None]
    at = (place[:, None] + col).clamp(max=pages - 1)
    i.table = torch.where(live, order[at], torch.full_like(order[at], -1)).contiguous()
    i.lens, i.rows, i.per = lens, rows, per
    i.refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    i.refs[i.table[live].long()] = 1
    if case["op"] == "fork":
        child = torch.arange(p, p + p * k, device="cuda", dtype=torch.int32)
        i.children = child[torch.randperm(p * k, generator=g, device="cuda")].contiguous()
        i.parents = torch.arange(p, device="cuda", dtype=torch.int32).repeat_interleave(k)
        i.room = torch.zeros(rows, dtype=torch.int32, device="cuda")
        i.room[p:] = 1
    i.pool, i.scale = _pool(case, g, pages)
    return i


class State:
    def __init__(self, case, seed):
        self.case = case
        op = case["op"]
        if op in ("fork", "compact"):
            self.__dict__.update(vars(_tables(case, seed)))
            if op == "compact":
                self.table_out, self.refs_out = torch.full_like(self.table, -1), torch.zeros_like(self.refs)
                self.n_used = torch.zeros(1, dtype=torch.int32, device="cuda")
        else:
            self.__dict__.update(vars(_cache(case, seed)))
            b, T, D, H, dh = (case[k] for k in ("batch", "T", "D", "heads", "d_head"))
            n = case["kv_heads"] * dh
            randn = lambda *s: torch.randn(*s, generator=self.g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
            if op == "write":
                self.w = randn(2, D, n) / math.sqrt(D)
                self.x = randn(b, T, D)
                self.values = torch.empty(self.kv.shape, dtype=torch.bfloat16, device="cuda")
            else:
                self.q = randn(b, T, H, dh) * case["q_scale"]
                self.out = torch.empty_like(self.q)
        self.ctx = None
        if own:
            self.handle()

    def handle(self):
        """The library's context, descriptors and workspace."""
        import paper_2410_03111_b200 as lorc
        L, case = lorc.load(), self.case
        self.L = L
        if case["op"] in ("fork", "compact"):
            self.ctx = L.lorc_create(1, 64, 1, 1, 64, 10000.0, max_pos=16)
            bufs = [self.pool[l, i] for l in range(case["layers"]) for i in range(2)]
            if self.scale is not None:
                bufs += [self.scale[l, i] for l in range(case["layers"]) for i in range(2)]
            self.pages = L.make_pages(bufs, self.table, self.lens, self.refs, self.page)
            need = L.lorc_pages_workspace_bytes(self.pages, self.rows)
        else:
            style = {"half": L.LORC_ROPE_HALF_SPLIT, "interleaved": L.LORC_ROPE_INTERLEAVED, "none": L.LORC_ROPE_NONE}
            b, n, dh = case["batch"], case["kv_heads"] * case["d_head"], case["d_head"]
            self.ctx = L.lorc_create(1, case["D"], case["heads"], case["kv_heads"], dh, case["theta"], rope_style=style[case["rope"]],
                                     max_pos=case["len_max"] + 64)
            w = self.w if case["op"] == "write" else torch.zeros(2, case["D"], n, dtype=torch.bfloat16, device="cuda")
            L.lorc_load_factors(self.ctx, 0, L.LORC_MODE_FULL, 0, 0, w[0], None, w[1], None)
            type = {"int8": L.LORC_CACHE8_INT8, "e4m3": L.LORC_CACHE8_E4M3}[case["type"]]
            where = dict(page_table=self.table, page_size=case["page"], max_pages_per_seq=self.table.shape[1],
                         n_pages=self.table.numel()) if case["page"] else dict(seq_stride=self.rows_per_page)
            self.cache = L.make_cache8(self.kv[0], self.kv[1], self.scale[0], self.scale[1], self.lens, b, case["len_max"], type, **where)
            need = L.lorc_cache8_workspace_bytes(self.ctx, b, case["len_max"], case["T"])
        self.ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
        L.lorc_set_workspace(self.ctx, self.ws)

    def __del__(self):
        if getattr(self, "ctx", None) is not None:
            torch.cuda.synchronize()
            self.L.lorc_destroy(self.ctx)
            self.ctx = None


def prepare(case, seed):
    return State(case, seed)


# ---- one pass --------------------------------------------------------------------------------------------------------------

def run(state):
    return {"write": _run_write, "decode": _run_decode, "chunk": _run_chunk, "fork": _run_fork, "compact": _run_compact}[state.case["op"]](state)


def _by_block(state, t):
    """[2, pages, page, n] as [2, pages, blocks, 16, kv_heads, d_head]"""
    c = state.case
    return t.view(2, t.shape[1], -1, BLOCK, c["kv_heads"], c["d_head"])


def _values(state):
    """The numbers that the cache stands for.  They fit bf16: a code has at most seven significant bits, scales are powers of two."""
    scale = state.scale[:, :, :, None, :, None]
    if state.case["type"] == "int8":
        torch.mul(_by_block(state, state.kv), scale, out=_by_block(state, state.values))
    else:
        state.values.copy_(state.kv)
        _by_block(state, state.values).mul_(scale)
    return {"values": state.values}


def _run_write(s):
    if own:
        s.L.lorc_append8(s.ctx, 0, s.cache, s.x, s.case["T"])
    else:
        _write(s)
    return _values(s)


def _run_decode(s):
    if own:
        s.L.lorc_decode_attn8(s.ctx, 0, s.cache, s.q, s.out)
        return {"out": s.out}
    return {"out": _attend(s)}


def _run_chunk(s):
    if own:
        s.L.lorc_prefill_attn8(s.ctx, 0, s.cache, s.q, s.out, s.case["T"])
        return {"out": s.out}
    return {"out": _attend(s)}


def _run_fork(s):
    if own:
        L = s.L
        L.lorc_pages_free(s.ctx, s.pages, s.children, s.children.numel())
        L.lorc_pages_fork(s.ctx, s.pages, s.parents, s.children, s.children.numel())
        L.lorc_pages_grow(s.ctx, s.pages, s.room)
    else:
        _free(s)
        _fork_pages(s)
        _grow(s)
    return {"pool": s.pool, "scale": s.scale, "table": s.table, "lens": s.lens, "refs": s.refs}


def _run_compact(s):
    if own:
        s.L.lorc_pages_compact(s.ctx, s.pages, s.table_out, s.refs_out, s.n_used)
    else:
        _compact_pages(s)
    return {"pool": s.pool, "scale": s.scale, "table": s.table_out, "refs": s.refs_out, "n_used": s.n_used}


# ---- plain forms -----------------------------------------------------------------------------------------------------------

def _rope(case, t, pos):
    """t [..., d_head] fp32 rotated at pos, which has t's leading dimensions but the heads'; the angles in fp64."""
    if case["rope"] == "none":
        return t
    d = case["d_head"]
    j = torch.arange(d // 2, device=t.device, dtype=torch.float64)
    angle = pos.double()[..., None, None] * case["theta"] ** (-2.0 * j / d)
    c, s = torch.cos(angle).float(), torch.sin(angle).float()
    if case["rope"] == "half":
        a, b = t[..., : d // 2], t[..., d // 2:]
        return torch.cat([a * c - b * s, a * s + b * c], -1)
    a, b = t[..., 0::2], t[..., 1::2]
    return torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)


def _row_of(state, pos):
    """Page and row in the page of positions pos [batch, ...]."""
    b, ps = pos.shape[0], state.rows_per_page
    seq = torch.arange(b, device="cuda").view(b, *[1] * (pos.dim() - 1)).expand_as(pos)
    page = state.table[seq, pos // ps].long() if state.table is not None else seq
    return page, pos % ps


def _round_codes(case, v):
    if case["type"] == "int8":
        return v.round().clamp(-127, 127).to(torch.int8)
    return v.clamp(-448, 448).to(torch.float8_e4m3fn)


def _write(s):
    c = s.case
    b, T, D, hkv, dh = (c[k] for k in ("batch", "T", "D", "kv_heads", "d_head"))
    new = (s.x.float().view(1, b * T, D) @ s.w.float()).view(2, b, T, hkv, dh)
    first = s.lens.long() - T
    new = torch.stack([_rope(c, new[0], first[:, None] + torch.arange(T, device="cuda")), new[1]])
    # the blocks that the new tokens reach, and what each of their rows is
    nb = (T + BLOCK - 2) // BLOCK + 1
    pos = (first // BLOCK * BLOCK)[:, None, None] + torch.arange(nb * BLOCK, device="cuda").view(nb, BLOCK)
    is_old, is_new = pos < first[:, None, None], (pos >= first[:, None, None]) & (pos < s.lens[:, None, None])
    page, row = _row_of(s, pos)
    block = row[:, :, 0] // BLOCK
    codes = s.kv.view(torch.uint8)[:, page, row].view(s.kv.dtype)                # [2, b, nb, 16, n]
    old = codes.float().view(2, b, nb, BLOCK, hkv, dh)
    old_scale = s.scale[:, page[:, :, 0], block]                                 # [2, b, nb, hkv]
    at = (pos - first[:, None, None]).clamp(0, T - 1)
    val = new[:, torch.arange(b, device="cuda")[:, None, None], at]              # [2, b, nb, 16, hkv, dh]
    val = torch.where(is_new[..., None, None], val, 0.0)
    # smallest e with amax <= largest 2^e (fp64: values next to a border)
    most = val.abs().amax(dim=(3, 5)).double()
    m, e = torch.frexp(most / LARGEST[c["type"]])
    e = torch.where(m == 0.5, e - 1, e).clamp(-100, 100)
    e = torch.where(most == 0, -100, e)
    need = torch.ldexp(torch.ones_like(most), e).float()
    has_old, has_new = is_old.any(-1)[..., None], is_new.any(-1)[..., None]
    scale = torch.where(has_old, torch.maximum(need, old_scale), need)
    scale = torch.where(has_new, scale, old_scale)
    per_row = scale[:, :, :, None, :, None]
    kept = torch.where(scale == old_scale, 1.0, old_scale / scale)[:, :, :, None, :, None]
    now = torch.where(is_new[..., None, None], val / per_row, old * kept)
    touched = (is_old | is_new) & has_new
    now = torch.where(touched[..., None], _round_codes(c, now).view(2, b, nb, BLOCK, hkv * dh).view(torch.uint8), codes.view(torch.uint8))
    s.kv.view(torch.uint8)[:, page, row] = now
    s.scale[:, page[:, :, 0], block] = scale


def _attend(s):
    c = s.case
    b, T, H, hkv, dh, N = c["batch"], c["T"], c["heads"], c["kv_heads"], c["d_head"], c["len_max"]
    pos = torch.arange(N, device="cuda").expand(b, N)
    page, row = _row_of(s, pos)
    first = s.lens.long() - T
    at = first[:, None] + torch.arange(T, device="cuda")                         # the queries' positions
    q = _rope(c, s.q.float(), at).view(b, T, hkv, H // hkv, dh)
    scale = s.scale[:, page, row // BLOCK]                                       # [2, b, N, hkv]
    k = s.kv[0].view(torch.uint8)[page, row].view(s.kv.dtype).float().view(b, N, hkv, dh) * scale[0][..., None]
    score = torch.einsum("btkgd,bnkd->bkgtn", q, k) / math.sqrt(dh)
    score.masked_fill_((pos[:, None, :] > at[:, :, None])[:, None, None], -math.inf)
    score -= score.amax(-1, keepdim=True)
    p = score.exp_()
    total = p.sum(-1)
    v = s.kv[1].view(torch.uint8)[page, row].view(s.kv.dtype).float().view(b, N, hkv, dh) * scale[1][..., None]
    out = torch.einsum("bkgtn,bnkd->btkgd", p, v) / total.permute(0, 3, 1, 2)[..., None]
    return out.reshape(b, T, H, dh).bfloat16()


def _held(s, rows, lens):
    """Which entries of the rows' tables hold pages, for each of lens tokens."""
    return torch.arange(s.per, device="cuda") < (-(-lens // s.page))[:, None]


def _free(s):
    rows = s.children.long()
    entries, live = s.table[rows], _held(s, rows, s.lens[rows])
    s.refs.index_add_(0, entries.clamp(min=0).flatten().long(), -live.flatten().int())
    s.lens[rows] = 0


def _lowest_free(s):
    """The free pages in ascending order (the entries behind them say nothing)."""
    free = s.refs == 0
    n = free.numel()
    listed = torch.zeros(n + 1, dtype=torch.long, device="cuda")
    listed.scatter_(0, torch.where(free, torch.cumsum(free, 0) - 1, n), torch.arange(n, device="cuda"))
    return listed


def _fork_pages(s):
    rows, child = s.parents.long(), s.children.long()
    lens = s.lens[rows]
    full, part = (lens // s.page).long(), lens % s.page > 0
    new = _lowest_free(s)[(torch.cumsum(part, 0) - 1).clamp(min=0)]
    entries, live = s.table[rows], _held(s, rows, lens)
    src = entries.gather(1, full[:, None].clamp(max=s.per - 1))[:, 0].long()
    here = part[:, None] & (torch.arange(s.per, device="cuda") == full[:, None])
    entries = torch.where(here, new[:, None].int(), entries)
    s.table[child] = torch.where(live, entries, s.table[child])
    s.refs.index_add_(0, entries.clamp(min=0).flatten().long(), live.flatten().int())
    s.lens[child] = lens
    # where no page is partly filled the first one is copied onto itself
    dst = torch.where(part, new, entries[:, 0].long())
    src = torch.where(part, src, entries[:, 0].long())
    s.pool[:, :, dst] = s.pool[:, :, src]
    if s.scale is not None:
        s.scale[:, :, dst] = s.scale[:, :, src]


def _grow(s):
    """Room for one token in some rows: a page where the last one is full."""
    more = (s.room > 0) & (s.lens % s.page == 0)
    new = _lowest_free(s)[(torch.cumsum(more, 0) - 1).clamp(min=0)]
    here = more[:, None] & (torch.arange(s.per, device="cuda") == (s.lens // s.page)[:, None])
    s.table.copy_(torch.where(here, new[:, None].int(), s.table))
    s.refs.index_add_(0, new, more.int())
    s.lens += s.room


def _compact_pages(s):
    used = s.refs > 0
    n = used.sum()
    index = torch.arange(used.numel(), device="cuda")
    dst, src = torch.nonzero(~used & (index < n))[:, 0], torch.nonzero(used & (index >= n))[:, 0]
    s.pool[:, :, dst] = s.pool[:, :, src]
    if s.scale is not None:
        s.scale[:, :, dst] = s.scale[:, :, src]
    to = index.clone()
    to[src] = dst
    rows = torch.arange(s.rows, device="cuda")
    s.table_out.copy_(torch.where(_held(s, rows, s.lens), to[s.table.clamp(min=0).long()].int(), s.table))
    s.refs_out.copy_(torch.where(index < n, s.refs, 0))
    s.refs_out[dst] = s.refs[src]
    s.n_used.copy_(n.int())


# ---- in 64 bits ------------------------------------------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] in ("fork", "compact"):
        return None                          # pages are moved, nothing is computed
    s = State(case, seed)
    return {"values": _exact_write(s)} if case["op"] == "write" else {"out": _exact_attention(s)}


def _rotation(case, pos):
    """Rotation matrices [positions, d_head, d_head] in fp64."""
    d, n = case["d_head"], pos.numel()
    if case["rope"] == "none":
        return torch.eye(d, dtype=torch.float64, device="cuda").expand(n, d, d)
    r = torch.zeros(n, d, d, dtype=torch.float64, device="cuda")
    j = torch.arange(d // 2, device="cuda")
    a, b = (j, j + d // 2) if case["rope"] == "half" else (2 * j, 2 * j + 1)
    angle = pos.double()[:, None] * torch.pow(torch.tensor(case["theta"], dtype=torch.float64, device="cuda"), -j.double() * 2 / d)
    r[:, a, a], r[:, b, b] = torch.cos(angle), torch.cos(angle)
    r[:, b, a], r[:, a, b] = torch.sin(angle), -torch.sin(angle)
    return r


def _exact_rows(s, seq, n):
    """Index of the first n tokens of a sequence into the flattened rows of the cache."""
    pos = torch.arange(n, device="cuda")
    if s.table is None:
        return seq * s.rows_per_page + pos
    return torch.cat([p * s.rows_per_page + torch.arange(s.rows_per_page, device="cuda") for p in s.table[seq].tolist()])[:n]


def _exact_write(s):
    c = s.case
    hkv, dh, T, top = c["kv_heads"], c["d_head"], c["T"], LARGEST[c["type"]]
    codes = s.kv.double().view(2, -1, hkv, dh)
    scales = s.scale.double().view(2, -1, hkv).clone()
    if c["type"] == "int8":
        rounded = lambda v: torch.round(v).clamp(-top, top)  # noqa: E731
    else:
        # three bits behind the leading one, exponents from -6 on
        def rounded(v):
            step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
            return (torch.round(v / step) * step).clamp(-top, top)
    for seq, n in enumerate(s.lens.tolist()):
        rows = _exact_rows(s, seq, n)
        new = s.x[seq].double() @ s.w.double()
        new = new.view(2, T, hkv, dh)
        pos = torch.arange(n - T, n, device="cuda")
        new[0] = torch.einsum("tij,thj->thi", _rotation(c, pos), new[0])
        for begin in range((n - T) // BLOCK * BLOCK, n, BLOCK):
            end, start = min(n, begin + BLOCK), max(begin, n - T)
            blk = rows[begin] // BLOCK
            fresh = new[:, start - (n - T): end - (n - T)]
            peak = fresh.abs().amax(dim=(1, 3))
            power = torch.exp2(torch.ceil(torch.log2(peak / top)).clamp(-100, 100))
            if start > begin:
                power = torch.maximum(power, scales[:, blk])
                codes[:, rows[begin:start]] = rounded(codes[:, rows[begin:start]] * (scales[:, blk] / power)[:, None, :, None])
            codes[:, rows[start:end]] = rounded(fresh / power[:, None, :, None])
            scales[:, blk] = power
    out = codes.view(2, -1, BLOCK, hkv, dh) * scales.view(2, -1, 1, hkv, 1)
    return out.view(s.kv.shape)


def _exact_attention(s):
    c = s.case
    hkv, dh, T, H = c["kv_heads"], c["d_head"], c["T"], c["heads"]
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    codes, scales = s.kv.view(2, -1, hkv, dh), s.scale.double().view(2, -1, hkv)
    for seq, n in enumerate(s.lens.tolist()):
        rows = _exact_rows(s, seq, n)
        k, v = (codes[i].view(torch.uint8)[rows].view(codes.dtype).double() * scales[i][rows // BLOCK][..., None] for i in (0, 1))
        pos = torch.arange(n - T, n, device="cuda")
        q = torch.einsum("tij,thj->thi", _rotation(c, pos), s.q[seq].double())
        later = torch.arange(n, device="cuda")[None, :] > pos[:, None]
        for h in range(H):
            kvh = h // (H // hkv)
            w = torch.softmax((q[:, h] @ k[:, kvh].T / math.sqrt(dh)).masked_fill(later, -math.inf), -1)
            out[seq, :, h] = w @ v[:, kvh]
    return out


# ---- work ------------------------------------------------------------------------------------------------------------------

def work(case):
    """Every input read once and every output written once: codes and scales, weights, tokens, queries, results, moved pages."""
    op = case["op"]
    if op in ("fork", "compact"):
        per_page = case["layers"] * 2 * case["page"] * case["width"] * (2 if case["form"] == "bf16" else 1)
        if case["form"] != "bf16":
            per_page += case["layers"] * 2 * case["page"] // BLOCK * (case["width"] // 128) * 4
        mean = (case["len_min"] + case["len_max"]) / 2
        if op == "fork":
            rows = case["parents"] * case["children"]
            moved, entries = rows * (1 - 1 / case["page"]), rows * mean / case["page"]
        else:
            used = max(1, int(case["rows"] * case["keep"])) * (mean / case["page"] + 0.5)
            moved, entries = used * max(0.0, 1 - used / case["pages"]), case["rows"] * -(-case["len_max"] // case["page"])
        return {"bytes": 2 * moved * per_page + 8 * entries + 8 * case["pages"], "flops": 0}
    b, T, D, H, dh, hkv = (case[k] for k in ("batch", "T", "D", "heads", "d_head", "kv_heads"))
    n, length = hkv * dh, (max(T, case["len_min"]) + case["len_max"]) / 2
    if op == "write":
        return {"bytes": 2 * b * T * D + 2 * D * 2 * n + b * T * 2 * n + 2 * b * -(-T // BLOCK) * hkv * 4, "flops": 2.0 * b * T * D * 2 * n}
    pairs = b * T * (length - (T - 1) / 2)
    return {"bytes": b * length * 2 * n + 2 * b * length / BLOCK * hkv * 4 + 2 * 2 * b * T * H * dh, "flops": 4.0 * pairs * H * dh}
