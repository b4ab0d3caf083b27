"""What the operators around the 4-bit key/value cache are measured on: rotating a step's queries and keys on their way into a paged cache
(bf16 or 4-bit), and the attention of a step over the 4-bit cache.

A case is a dict of plain values:
  entry            "append": rotate, and append to a bf16 pool.  "append4": rotate, quantise and append to a 4-bit pool, then read the
                   new tokens back as the values that the cache holds.  "attention4": the attention of a step over a 4-bit pool
  hq, hkv, d       q-heads, kv-heads, head dimension (page size is always 16)
  rot, interleaved rotated dimensions of a head (0: none), and whether pairs are neighbours or half of the rotated dimensions apart
  packed           whether queries, keys and values come as the rows of one buffer (the output of one projection) or apart
  decodes, ctx_lo, ctx_hi, log
                   that many decode requests, contexts spread over [ctx_lo, ctx_hi], evenly over the logarithm if `log`
  prompts          prompt chunks as "chunk+prior" tokens, comma separated
  lengths          the seed the lengths are drawn with (they belong to the case, values to `prepare`'s seed)

The 4-bit pool is uint8 [page][kv-head][17 d]: of the 16 tokens of a page and a head the codes of the keys [16][d/32][16], those of the values
[2][d/64][16][2][8], the scales of the keys [16][d/32] and of the values [2][d/64][8][2].  A byte of the keys holds two neighbouring dimensions
of a block of 32, a byte of the values dimensions i and i + 16 of one, the lower one in the low four bits; codes are sign and E2M1 magnitude, scales
exponents of two plus 127.
"""
import functools
import math

import numpy as np
import torch

own = False

PAGE = 16
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
# head layouts (q-heads, kv-heads, head dimension) of the drawn cases
LAYOUTS = ((32, 8, 128), (32, 8, 128), (8, 1, 128), (8, 2, 128), (8, 8, 128), (24, 8, 128), (32, 8, 64), (32, 4, 64))


def _case(entry, hq, hkv, d, rot=0, interleaved=False, packed=True, decodes=0, ctx_lo=0, ctx_hi=0, log=False, prompts="", lengths=0, name=None):
    c = dict(entry=entry, hq=hq, hkv=hkv, d=d, rot=rot, interleaved=interleaved, packed=packed, decodes=decodes, ctx_lo=ctx_lo, ctx_hi=ctx_hi,
             log=log, prompts=prompts, lengths=lengths)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one layer of a lightly loaded instance: the new tokens of four decodes; launches are all that counts
        _case("append", 32, 8, 128, 128, decodes=4, ctx_lo=100, ctx_hi=2000, log=True, lengths=1, name="append_few"),
        # one layer of a step with long prompt chunks beside decodes: bound by memory
        _case("append", 32, 8, 128, 128, decodes=32, ctx_lo=1792, ctx_hi=2304, prompts="2048+0,2048+4096,2048+8192,2048+12285", lengths=4,
              name="append_chunks"),
        # one kv-head per q-head, 64 wide, a quarter rotated in neighbouring pairs, odd chunks that begin and end inside pages, tensors apart
        _case("append", 8, 8, 64, 16, True, False, decodes=21, ctx_lo=150, ctx_hi=6000, prompts="301+0,1029+700,130+63", lengths=8,
              name="append_d64_partial"),
        # the new tokens of a large decode batch go into the 4-bit cache, one to a page
        _case("append4", 32, 8, 128, 128, decodes=256, ctx_lo=2048, ctx_hi=16384, lengths=3, name="append4_decodes"),
        # long prompt chunks into the 4-bit cache: bound by memory
        _case("append4", 32, 8, 128, 128, decodes=32, ctx_lo=1792, ctx_hi=2304, prompts="2048+0,2048+4096,2048+8192,2048+12285", lengths=4,
              name="append4_chunks"),
        # 64-wide heads, odd chunks, neighbouring pairs
        _case("append4", 32, 8, 64, 64, True, decodes=48, ctx_lo=150, ctx_hi=6000, log=True, prompts="301+0,1029+700,130+63", lengths=8,
              name="append4_d64"),
        # one layer of a lightly loaded instance: a few decodes, latency
        _case("attention4", 32, 8, 128, decodes=4, ctx_lo=100, ctx_hi=2000, log=True, lengths=1, name="attention4_few"),
        # one layer of a large decode batch: bound by HBM
        _case("attention4", 32, 8, 128, decodes=256, ctx_lo=2048, ctx_hi=16384, lengths=3, name="attention4_decodes"),
        # one layer of a step with long prompt chunks on grown contexts: bound by the matrix cores
        _case("attention4", 32, 8, 128, decodes=32, ctx_lo=1792, ctx_hi=2304, prompts="2048+0,2048+4096,2048+8192,2048+12288", lengths=4,
              name="attention4_prompts"),
        # a tensor-parallel share of a large layer at long contexts: one kv-head for eight q-heads
        _case("attention4", 8, 1, 128, decodes=16, ctx_lo=32768, ctx_hi=131072, prompts="4096+61440", lengths=5, name="attention4_long"),
        # the prefill of a single odd-sized prompt
        _case("attention4", 32, 8, 128, prompts="777+0", lengths=7, name="attention4_prompt"),
        # 64-wide heads, odd lengths of both kinds
        _case("attention4", 32, 8, 64, decodes=48, ctx_lo=150, ctx_hi=6000, log=True, prompts="301+0,1029+700,130+63", lengths=8,
              name="attention4_d64"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    entry = rng.choice(("append", "append4", "attention4", "attention4"))
    hq, hkv, d = rng.choice(LAYOUTS)
    rot, interleaved, packed = 0, False, True
    if entry != "attention4":
        rot, interleaved, packed = rng.choice((d, d, d, d // 2, 32, 16, 0)), rng.random() < 0.4, rng.random() < 0.6
    kind = rng.choice(("decode", "prefill", "mixed"))
    decodes = ctx_lo = ctx_hi = 0
    if kind != "prefill":
        decodes = _log_int(rng, 1, 256)
        ctx_hi = _log_int(rng, 1, max(2, min(131072, (2300000 if kind == "decode" and entry == "attention4" else 400000) // decodes)))
        ctx_lo = _log_int(rng, 1, ctx_hi)
    chunks = []
    if kind != "decode":
        room, rows = 4.5e11, 8192      # multiply-adds and rows of all chunks together: no more than the largest listed cases
        for _ in range(rng.randint(1, 6)):
            q, prior = _log_int(rng, 2, 4096), rng.choice((0, 0, _log_int(rng, 1, 16384), _log_int(rng, 16, 65536)))
            work = 2 * d * hq * (q * prior + q * (q + 1) / 2)
            if work <= room and q <= rows:
                chunks.append(f"{q}+{prior}")
                room -= work
                rows -= q
        if not chunks:
            chunks = ["333+100"]
    return _case(entry, hq, hkv, d, rot, interleaved, packed, decodes, ctx_lo, ctx_hi, rng.random() < 0.5, ",".join(chunks), rng.randrange(1 << 30))


@functools.lru_cache(maxsize=64)
def _lengths_of(decodes, ctx_lo, ctx_hi, log, prompts, lengths):
    g = np.random.default_rng(lengths)
    kind, q, c = [], [], []
    if decodes:
        if log:
            ctx = np.rint(np.exp(g.uniform(math.log(ctx_lo), math.log(ctx_hi), decodes))).astype(np.int64)
        else:
            ctx = g.integers(ctx_lo, ctx_hi + 1, decodes)
        for n in ctx:
            kind.append(0); q.append(1); c.append(int(n))
    for item in prompts.split(",") if prompts else ():
        chunk, prior = item.split("+")
        kind.append(1); q.append(int(chunk)); c.append(int(chunk) + int(prior))
    return tuple(np.array(a, np.int32) for a in (kind, q, c))


def _lengths(case):
    """kind (0 a decode, 1 a prompt chunk), q_len, ctx_len of the step's requests."""
    return _lengths_of(*(case[k] for k in ("decodes", "ctx_lo", "ctx_hi", "log", "prompts", "lengths")))


def _positions(q_len, ctx_len):
    return np.concatenate([np.arange(c - q, c) for q, c in zip(q_len.tolist(), ctx_len.tolist())])


# ---------------------------------------------------------------- the 4-bit format, plainly
def _quantise(x):
    """fp32 [..., D] -> codes uint8 [..., D], scale bytes uint8 [..., D / 32]."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = b.abs().amax(-1).view(torch.int32)
    e = (((top + 0x200000) >> 23) - 2).clamp(2, 252)
    y = b * ((254 - e) << 23).view(torch.float32)[..., None]
    m = y.abs()
    code = (m > 0.25).to(torch.uint8)
    for limit, even_below in ((0.75, False), (1.25, True), (1.75, False), (2.5, True), (3.5, False), (5.0, True)):
        code += (m > limit) if even_below else (m >= limit)
    code += 8 * torch.signbit(y).to(torch.uint8)
    return code.reshape(x.shape), torch.where(top >= 0x7F800000, 255, e).to(torch.uint8)


def _value(code, e):
    """codes [..., D], scale bytes [..., D / 32] -> fp32 [..., D]."""
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=code.device)
    scale = torch.where(e == 255, math.nan, torch.exp2(e.float() - 127.0))
    return (table[code.long()].reshape(*code.shape[:-1], -1, 32) * scale[..., None]).reshape(code.shape)


def _sections(pool, d):
    """Views of a pool: key codes, value codes, key scales, value scales."""
    p, h = pool.shape[:2]
    return (pool[:, :, :8 * d].view(p, h, PAGE, d // 32, 16), pool[:, :, 8 * d:16 * d].view(p, h, 2, d // 64, 16, 2, 8),
            pool[:, :, 16 * d:16 * d + d // 2].view(p, h, PAGE, d // 32), pool[:, :, 16 * d + d // 2:].view(p, h, 2, d // 64, 8, 2))


def _put(pool, page, slot, k, v, d):
    """Tokens [n, heads, d] in fp32 go to slots of pages."""
    key, value, key_scale, value_scale = _sections(pool, d)
    n, h = k.shape[:2]
    code, e = _quantise(k)
    code = code.view(n, h, d // 32, 16, 2)
    key[page, :, slot] = code[..., 0] | code[..., 1] << 4
    key_scale[page, :, slot] = e
    code, e = _quantise(v)
    code = code.view(n, h, d // 64, 2, 2, 16).permute(0, 1, 2, 5, 3, 4)               # [n, h, d/64, 16, 2, low or high]
    half, at = slot // 8, slot % 8
    value[page, :, half, :, :, :, at] = code[..., 0] | code[..., 1] << 4
    value_scale[page, :, half, :, at] = e.view(n, h, d // 64, 2)


def _get(pages, d):
    """Whole pages [n, heads, 17 d] -> keys and values fp32 [n, heads, 16, d]."""
    key, value, key_scale, value_scale = _sections(pages, d)
    n, h = pages.shape[:2]
    k = _value(torch.stack((key & 15, key >> 4), -1).reshape(n, h, PAGE, d), key_scale)
    code = torch.stack((value & 15, value >> 4), -1)                                  # [n, h, 2, d/64, 16, 2, 8, low or high]
    v = _value(code.permute(0, 1, 2, 6, 3, 5, 7, 4).reshape(n, h, PAGE, d), value_scale.permute(0, 1, 2, 4, 3, 5).reshape(n, h, PAGE, d // 32))
    return k, v


# ---------------------------------------------------------------- inputs
def _inputs(case, seed):
    """The step's arrays: lengths and block table on the host, values and, for the plain form, indices on the GPU."""
    kind, q_len, ctx_len = _lengths(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    g = np.random.default_rng([seed, 1])
    n_pages = (ctx_len.astype(np.int64) + PAGE - 1) // PAGE
    indptr = np.zeros(len(kind) + 1, np.int32)
    indptr[1:] = np.cumsum(n_pages)
    need = int(indptr[-1])
    num_pages = max(1, -(-need * 5 // 4))
    pages = g.permutation(num_pages)[:need].astype(np.int32)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    tokens = int(q_len.sum())
    s = {"case": case, "kind": kind, "q_len": q_len, "ctx_len": ctx_len, "indptr": indptr, "pages": pages, "num_pages": num_pages}
    # keys have channels of different size, some of them much larger than the others
    channel = torch.exp(0.4 * torch.empty((hkv, d), device="cuda").normal_(generator=gen))
    channel[:, 3::41] *= 3.0
    if case["entry"] == "append":
        s["pool"] = normal(num_pages, hkv, 2, PAGE * d)
    else:
        s["pool"] = torch.empty((num_pages, hkv, 17 * d), dtype=torch.uint8, device="cuda")
        slots = torch.arange(PAGE, device="cuda")
        step = max(1, (1 << 25) // (hkv * PAGE * d))
        for a in range(0, num_pages, step):
            n = min(step, num_pages - a)
            k, v = normal(n * PAGE, hkv, d).float() * channel, normal(n * PAGE, hkv, d).float()
            _put(s["pool"], torch.arange(a, a + n, device="cuda").repeat_interleave(PAGE), slots.repeat(n), k, v, d)
    if case["entry"] == "attention4":
        s["q"] = normal(tokens, hq, d)
        return s
    if case["packed"]:
        s["qkv"] = normal(tokens, (hq + 2 * hkv) * d)
        q, k, v = s["qkv"].split((hq * d, hkv * d, hkv * d), 1)
    else:
        q, k, v = normal(tokens, hq * d), normal(tokens, hkv * d), normal(tokens, hkv * d)
    k *= channel.reshape(-1)
    s["q"], s["k"], s["v"] = q, k, v
    if case["rot"]:
        # the model's table of rotations: a row for each position, cosines and then sines
        half = case["rot"] // 2
        rows = max(1024, -(-int(ctx_len.max()) // 1024) * 1024)
        angle = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * 500000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        s["cos_sin"] = torch.cat((angle.cos(), angle.sin()), 1).float()
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    q_len, ctx_len, indptr, pages = s["q_len"], s["ctx_len"], s["indptr"], s["pages"]
    tokens = int(q_len.sum())
    if not own:
        position = _positions(q_len, ctx_len)
        request = np.repeat(np.arange(len(q_len)), q_len)
        s["position"] = torch.from_numpy(position).cuda()
        s["page"] = torch.from_numpy(pages[indptr[request] + position // PAGE].astype(np.int64)).cuda()
        s["slot"] = s["position"] % PAGE
        s["ids"] = [torch.from_numpy(pages[indptr[r]:indptr[r + 1]].astype(np.int64)).cuda() for r in range(len(q_len))]
        return s
    # the step's descriptor serves every layer of the step
    from paper_2508_15919_amd import binding as hb
    s["hb"], stream = hb, torch.cuda.current_stream()
    s["shape"] = hb.make_shape(case["hq"], case["hkv"], case["d"], s["num_pages"])
    host_bytes, device_bytes, ws_bytes = hb.hfx_batch_desc_sizes(s["shape"], s["kind"], q_len, ctx_len)
    s["host_desc"] = torch.empty(host_bytes, dtype=torch.uint8, pin_memory=True)
    s["device_desc"] = torch.empty(device_bytes, dtype=torch.uint8, device="cuda")
    hb.hfx_build_batch_desc(s["shape"], s["kind"], q_len, ctx_len, indptr, pages, s["host_desc"], s["device_desc"], stream)
    s["out"] = torch.empty((tokens, case["hq"], case["d"]), dtype=torch.bfloat16, device="cuda")
    if case["entry"] == "attention4":
        s["workspace"] = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda") if ws_bytes else None
        return s
    s["rope"] = hb.make_rope(s["cos_sin"], case["rot"], case["interleaved"]) if case["rot"] else None
    if case["entry"] == "append4":
        s["k_out"] = torch.empty((tokens, case["hkv"], case["d"]), dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.empty_like(s["k_out"])
    return s


# ---------------------------------------------------------------- one pass
def _rotated(s, x, heads):
    """Rows [tokens, heads * d] in bf16 -> fp32 [tokens, heads, d], rotated by their positions."""
    case = s["case"]
    x = x.float().view(x.shape[0], heads, case["d"]) if x.is_contiguous() else x.float().reshape(x.shape[0], heads, case["d"])
    rot, half = case["rot"], case["rot"] // 2
    if not rot:
        return x
    row = s["cos_sin"][s["position"]]
    c, t = row[:, None, :half], row[:, None, half:]
    if case["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        a, b = x[..., :half], x[..., half:rot]
    y = x.clone()
    first, second = a * c - b * t, b * c + a * t
    if case["interleaved"]:
        y[..., 0:rot:2], y[..., 1:rot:2] = first, second
    else:
        y[..., :half], y[..., half:rot] = first, second
    return y


def _plain_append(s):
    case, pool, page, slot = s["case"], s["pool"], s["page"], s["slot"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    q = _rotated(s, s["q"], hq).to(torch.bfloat16)
    k, v = _rotated(s, s["k"], hkv), s["v"].reshape(-1, hkv, d)
    if case["entry"] == "append":
        n = pool.shape[0]
        pool.view(n, hkv, 2, d // 16, PAGE, 16)[:, :, 0][page, :, :, slot] = k.to(torch.bfloat16).view(-1, hkv, d // 16, 16)
        pool.view(n, hkv, 2, d, PAGE)[:, :, 1][page, :, :, slot] = v
        return q, pool
    _put(pool, page, slot, k, v.float(), d)
    key, value = _get(pool[page], d)
    at = torch.arange(len(slot), device="cuda")
    return q, key[at, :, slot].to(torch.bfloat16), value[at, :, slot].to(torch.bfloat16)


def _plain_attention(s):
    case, q = s["case"], s["q"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    group, scale = hq // hkv, 1.0 / math.sqrt(d)
    out = torch.empty_like(q)
    t0 = 0
    for ids, n, q_len in zip(s["ids"], s["ctx_len"].tolist(), s["q_len"].tolist()):
        k, v = (x.permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :n] for x in _get(s["pool"][ids], d))
        rows = max(1, (1 << 28) // (n * hq))                     # chunk rows at a time: scores of a gigabyte
        for a in range(0, q_len, rows):
            b = min(q_len, a + rows)
            m = n - q_len + b                                    # keys that the last of these rows sees
            x = q[t0 + a:t0 + b].float().view(b - a, hkv, group, d).permute(1, 2, 0, 3).reshape(hkv, group * (b - a), d)
            w = (x @ k[:, :m].transpose(1, 2)).view(hkv, group, b - a, m) * scale
            if b - a > 1:
                hidden = torch.arange(m, device="cuda")[None, :] > torch.arange(n - q_len + a, m, device="cuda")[:, None]
                w.masked_fill_(hidden, -math.inf)
            w = torch.exp(w - w.amax(-1, keepdim=True))
            w /= w.sum(-1, keepdim=True)
            y = w.view(hkv, group * (b - a), m) @ v[:, :m]
            out[t0 + a:t0 + b] = y.view(hkv, group, b - a, d).permute(2, 0, 1, 3).reshape(b - a, hq, d)
        t0 += q_len
    return out


def run(s):
    case = s["case"]
    if not own:
        return _plain_attention(s) if case["entry"] == "attention4" else _plain_append(s)
    hb, stream = s["hb"], torch.cuda.current_stream()
    if case["entry"] == "attention4":      # one layer of a step whose descriptor is on the GPU
        hb.hfx_mixed_paged_attention_mx(s["shape"], s["q"], s["pool"], s["host_desc"], s["device_desc"], s["workspace"], s["out"], stream)
        return s["out"]
    q, k, v = s["q"], s["k"], s["v"]
    append = hb.hfx_rope_append_kv if case["entry"] == "append" else hb.hfx_rope_append_kv_mx
    append(s["shape"], s["rope"], q, q.stride(0), k, k.stride(0), v, v.stride(0), s["out"], s["pool"], s["host_desc"], s["device_desc"], stream)
    if case["entry"] == "append":
        return s["out"], s["pool"]
    hb.hfx_read_new_kv_mx(s["shape"], s["pool"], s["host_desc"], s["device_desc"], s["k_out"], s["v_out"], stream)
    return s["out"], s["k_out"], s["v_out"]


def work(case):
    kind, q, c = (a.astype(np.int64) for a in _lengths(case))
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    tokens = int(q.sum())
    if case["entry"] == "attention4":
        pairs = int((q * (c - q) + q * (q + 1) // 2).sum())          # visible (row, key) pairs
        return {"bytes": int(c.sum()) * hkv * d * 17 // 16 + 2 * tokens * hq * d * 2, "flops": 4 * d * hq * pairs}
    table = 4 * case["rot"] * len(np.unique(_positions(q, c)))
    rows = tokens * d * 2 * (2 * hq + 2 * hkv) + table               # queries in and out, keys and values in
    new = tokens * hkv * d * 4                                       # keys and values in bf16
    nbytes = rows + (new if case["entry"] == "append" else tokens * hkv * d * 17 // 16 + new)
    return {"bytes": nbytes, "flops": 3 * case["rot"] * tokens * (hq + hkv)}


# ---------------------------------------------------------------- in 64 bits, from the definition
def _exact_rotation(case, x, table, position, steps):
    """steps: round products and sums to 32 bits, as the operator does ahead of a format in which a value near a tie may go either way."""
    x = x.double()
    y = x.clone()
    m = case["rot"] // 2

    def r(z):
        return z.float().double() if steps else z
    for i in range(m):
        a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + m)
        c, t = table[position, i, None].double(), table[position, m + i, None].double()
        y[:, :, a] = r(r(x[:, :, a] * c) - r(x[:, :, b] * t))
        y[:, :, b] = r(r(x[:, :, b] * c) + r(x[:, :, a] * t))
    return y


def _exact_quantised(x):
    """What the 4-bit cache makes of values [tokens, heads, d]: of each 32 the smallest power of two under which the largest is nearest
    to a magnitude of at most 6, then the nearest magnitudes, those with an even code from halfway."""
    b = x.unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    exponent = torch.frexp(top)[1].double() - 1                        # top = [1, 2) * 2^exponent
    exponent = exponent - 2 + (top >= 1.75 * torch.exp2(exponent))
    scale = torch.exp2(torch.where(top > 0, exponent, -125.0).clamp(-125, 125))
    y = (b / scale).abs()
    grid = torch.tensor(MAGNITUDES, dtype=torch.float64, device=x.device)
    upper = torch.searchsorted(grid, y.contiguous()).clamp(1, 7)
    lower = upper - 1
    middle = (grid[lower] + grid[upper]) / 2
    index = torch.where((y > middle) | ((y == middle) & (upper % 2 == 0)), upper, lower)
    return (grid[index] * scale * torch.where(b < 0, -1.0, 1.0)).flatten(-2)


def exact(case, seed):
    s = _inputs(case, seed)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["entry"] != "attention4":
        position = torch.from_numpy(_positions(s["q_len"], s["ctx_len"])).cuda()
        q, k, v = (x.unflatten(1, (-1, d)) for x in (s["q"], s["k"], s["v"]))
        turned = _exact_rotation(case, q, s.get("cos_sin"), position, False)
        if case["entry"] == "append4":
            return turned, _exact_quantised(_exact_rotation(case, k, s.get("cos_sin"), position, True)), _exact_quantised(v.double())
        k = _exact_rotation(case, k, s.get("cos_sin"), position, False)
        pool = s["pool"].double()
        start = 0
        slot = torch.arange(PAGE, device="cuda")
        for r, (n, c) in enumerate(zip(s["q_len"].tolist(), s["ctx_len"].tolist())):
            for i in range((c - n) // PAGE, -(-c // PAGE)):            # the pages that get new tokens
                lo, hi = max(c - n - i * PAGE, 0), min(c - i * PAGE, PAGE)
                row = start + i * PAGE + lo - (c - n)
                block = pool[int(s["pages"][s["indptr"][r] + i])]
                block[:, 0].view(hkv, d // 16, PAGE, 16)[:, :, slot[lo:hi]] = k[row:row + hi - lo].permute(1, 0, 2).reshape(hkv, hi - lo, d // 16, 16).transpose(1, 2)
                block[:, 1].view(hkv, d, PAGE)[:, :, slot[lo:hi]] = v[row:row + hi - lo].double().permute(1, 2, 0)
            start += n
        return turned, pool
    out = torch.empty((len(s["q"]), hq, d), dtype=torch.float64, device="cuda")
    grid = torch.tensor(MAGNITUDES, dtype=torch.float64, device="cuda")

    def number(code):
        return grid[(code & 7).long()] * (1.0 - 2.0 * (code >> 3).double())
    t0 = 0
    for r, (q_len, n) in enumerate(zip(s["q_len"].tolist(), s["ctx_len"].tolist())):
        block = s["pool"][torch.from_numpy(s["pages"][s["indptr"][r]:s["indptr"][r + 1]].astype(np.int64)).cuda()]
        for g in range(hkv):
            key, value, ks, vs = (x[:, 0] for x in _sections(block[:, g:g + 1], d))
            k = torch.empty((len(block), PAGE, d), dtype=torch.float64, device="cuda")
            v = torch.empty_like(k)
            for w in range(d // 32):
                size = torch.exp2(ks[:, :, w].double() - 127)[..., None]
                k[:, :, 32 * w:32 * w + 32:2] = number(key[:, :, w] & 15) * size
                k[:, :, 32 * w + 1:32 * w + 32:2] = number(key[:, :, w] >> 4) * size
                byte = value[:, :, w // 2, :, w % 2].transpose(2, 3).reshape(-1, PAGE, 16)       # [pages, token, 16]
                size = torch.exp2(vs[:, :, w // 2, :, w % 2].reshape(-1, PAGE).double() - 127)[..., None]
                v[:, :, 32 * w:32 * w + 16] = number(byte & 15) * size
                v[:, :, 32 * w + 16:32 * w + 32] = number(byte >> 4) * size
            k, v = k.reshape(-1, d)[:n], v.reshape(-1, d)[:n]
            rows = max(1, (1 << 26) // n)
            for a in range(0, q_len, rows):
                b = min(q_len, a + rows)
                m = n - q_len + b
                hidden = torch.arange(m, device="cuda")[None, :] > torch.arange(n - q_len + a, m, device="cuda")[:, None]
                for h in range(g * (hq // hkv), (g + 1) * (hq // hkv)):
                    score = (s["q"][t0 + a:t0 + b, h].double() @ k[:m].T) / math.sqrt(d)
                    if b - a > 1:
                        score.masked_fill_(hidden, -math.inf)
                    out[t0 + a:t0 + b, h] = torch.softmax(score, dim=1) @ v[:m]
        t0 += q_len
    return out
