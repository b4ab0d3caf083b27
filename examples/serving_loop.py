"""A small serving loop over the page pool, held in bf16 or in 4 bits.

A decoder with random weights serves a queue of prompts: `hfx_compose_step` admits prompts beside the running requests' next tokens, one descriptor
is built per step and used by every layer, and each layer runs its projection, `hfx_rope_append_kv(_mx)` (rotation, queries packed, keys and values into
their pages) and `hfx_mixed_paged_attention(_mx)`.  Both pools serve the same requests; the second takes the tokens that the first chose, so that their
logits can be compared.  With `--weights 8` the projections are those of `hfx_matmul_rows`: weights and the rows that meet them in 8 bits, which `hfx_rms_norm`
(with the residual's addition) and `hfx_quantise_rows` (attention's rows, the activation) write.

    python examples/serving_loop.py                      # 2 layers of 32 / 8 heads of 128, 24 prompts, 32 tokens each
    python examples/serving_loop.py --layers 4 --requests 64 --new-tokens 64
    python examples/serving_loop.py --weights 8
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2508_15919_amd import binding as hb  # noqa: E402

PAGE = 16


class Decoder:
    """Weights of a decoder of `layers` layers: RMS norm, attention, RMS norm, two-matrix feed-forward; tied embedding."""

    def __init__(self, hq, hkv, d, layers, vocab, max_positions, seed=0):
        self.hq, self.hkv, self.d, self.layers = hq, hkv, d, layers
        hidden = hq * d
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(rows, cols, size):
            return torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda").normal_(0.0, size, generator=gen)
        self.embedding = normal(vocab, hidden, 1.0)
        self.qkv = [normal((hq + 2 * hkv) * d, hidden, hidden ** -0.5) for _ in range(layers)]
        self.out = [normal(hidden, hidden, hidden ** -0.5) for _ in range(layers)]
        self.up = [normal(2 * hidden, hidden, hidden ** -0.5) for _ in range(layers)]
        self.down = [normal(hidden, 2 * hidden, (2 * hidden) ** -0.5) for _ in range(layers)]
        angle = torch.arange(max_positions, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(d // 2, device="cuda", dtype=torch.float64) / (d // 2))
        self.rope = hb.make_rope(torch.cat((angle.cos(), angle.sin()), 1).float(), d)


class Weights8:
    """A decoder's weights in 8 bits, a scale for each output channel, and its norms."""

    def __init__(self, model):
        hidden, stream = model.hq * model.d, torch.cuda.current_stream()

        def handle(weight):
            n, k = weight.shape
            codes, scales = torch.empty((n, k), dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
            hb.hfx_quantise_rows(hb.HFX_ACT_NONE, n, k, weight, k, None, 0, None, codes, scales, stream)
            return hb.make_weight_q8(codes, scales)
        self.qkv, self.out, self.up, self.down = ([handle(w) for w in ws] for ws in (model.qkv, model.out, model.up, model.down))
        self.embedding = handle(model.embedding)
        self.norm = hb.make_norm(torch.ones(hidden, dtype=torch.bfloat16, device="cuda"), 1e-6)


def norm(x):
    y = x.float()
    return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)).to(torch.bfloat16)


class Cache:
    """The page pools of a decoder's layers, and the pages that are free."""

    def __init__(self, model, num_pages, four_bits):
        self.shape = hb.make_shape(model.hq, model.hkv, model.d, num_pages)
        self.four_bits = four_bits
        size = hb.hfx_mx_pool_bytes(self.shape) if four_bits else num_pages * model.hkv * 2 * PAGE * model.d * 2
        self.pools = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(model.layers)]
        self.append = hb.hfx_rope_append_kv_mx if four_bits else hb.hfx_rope_append_kv
        self.attend = hb.hfx_mixed_paged_attention_mx if four_bits else hb.hfx_mixed_paged_attention
        self.free = list(range(num_pages))[::-1]


class Step:
    """What the layers of a step share: its descriptor and workspace."""

    def __init__(self, cache, kind, q_len, ctx_len, pages):
        host, device, workspace = hb.hfx_batch_desc_sizes(cache.shape, kind, q_len, ctx_len)
        self.host = torch.empty(host, dtype=torch.uint8, pin_memory=True)
        self.device = torch.empty(device, dtype=torch.uint8, device="cuda")
        self.workspace = torch.empty(workspace, dtype=torch.uint8, device="cuda") if workspace else None
        indptr = np.concatenate(([0], np.cumsum([len(p) for p in pages]))).astype(np.int32)
        hb.hfx_build_batch_desc(cache.shape, kind, q_len, ctx_len, indptr, np.concatenate(pages).astype(np.int32), self.host, self.device,
                                torch.cuda.current_stream())


def forward(model, cache, step, tokens, last_rows, held=None):
    """Logits of the rows `last_rows` of a step with the packed tokens `tokens`; `held`: list that takes how far the first layer's values are off in the pool."""
    stream = torch.cuda.current_stream()
    hq, hkv, d = model.hq, model.hkv, model.d
    x = model.embedding[tokens]
    q = torch.empty((len(tokens), hq, d), dtype=torch.bfloat16, device="cuda")
    attended = torch.empty_like(q)
    for layer in range(model.layers):
        qkv = norm(x) @ model.qkv[layer].T                        # a token's queries, keys and values lie in one row
        qs, ks, vs = qkv.split((hq * d, hkv * d, hkv * d), 1)
        cache.append(cache.shape, model.rope, qs, qs.stride(0), ks, ks.stride(0), vs, vs.stride(0), q, cache.pools[layer], step.host, step.device, stream)
        if held is not None and layer == 0 and cache.four_bits:
            k_now, v_now = torch.empty((2, len(tokens), hkv, d), dtype=torch.bfloat16, device="cuda")
            hb.hfx_read_new_kv_mx(cache.shape, cache.pools[layer], step.host, step.device, k_now, v_now, stream)
            v = vs.float().reshape(v_now.shape)
            held.append(float((v_now.float() - v).norm() / v.norm()))
        cache.attend(cache.shape, q, cache.pools[layer], step.host, step.device, step.workspace, attended, stream)
        x = x + attended.reshape(len(tokens), hq * d) @ model.out[layer].T
        x = x + torch.nn.functional.silu(norm(x) @ model.up[layer].T) @ model.down[layer].T
    return norm(x[last_rows]).float() @ model.embedding.float().T


def forward_8(model, weights, cache, step, tokens, last_rows):
    """`forward` with the projections in 8 bits."""
    stream = torch.cuda.current_stream()
    hq, hkv, d, n = model.hq, model.hkv, model.d, len(tokens)
    hidden = hq * d

    def rows(cols, dtype=torch.bfloat16, count=n):
        return torch.empty((count, cols), dtype=dtype, device="cuda")
    x = model.embedding[tokens]
    q, attended, qkv, up, added = rows(hidden), rows(hidden), rows((hq + 2 * hkv) * d), rows(2 * hidden), rows(hidden)
    codes, wide_codes, scales = rows(hidden, torch.int8), rows(2 * hidden, torch.int8), torch.empty(n, device="cuda")
    qs, ks, vs = qkv.split((hidden, hkv * d, hkv * d), 1)

    def product(weight, codes, k, out):
        hb.hfx_matmul_rows(weight, n, codes, k, scales, out, out.shape[1], False, stream)
    for layer in range(model.layers):
        if layer == 0:
            hb.hfx_rms_norm(weights.norm, n, x, hidden, None, 0, None, None, codes, scales, stream)
        else:
            hb.hfx_rms_norm(weights.norm, n, added, hidden, x, hidden, x, None, codes, scales, stream)      # x takes what the layer before added
        product(weights.qkv[layer], codes, hidden, qkv)
        cache.append(cache.shape, model.rope, qs, qs.stride(0), ks, ks.stride(0), vs, vs.stride(0), q, cache.pools[layer], step.host, step.device, stream)
        cache.attend(cache.shape, q, cache.pools[layer], step.host, step.device, step.workspace, attended, stream)
        hb.hfx_quantise_rows(hb.HFX_ACT_NONE, n, hidden, attended, hidden, None, 0, None, codes, scales, stream)
        product(weights.out[layer], codes, hidden, added)
        hb.hfx_rms_norm(weights.norm, n, added, hidden, x, hidden, x, None, codes, scales, stream)
        product(weights.up[layer], codes, hidden, up)
        hb.hfx_quantise_rows(hb.HFX_ACT_SILU, n, 2 * hidden, up, 2 * hidden, None, 0, None, wide_codes, scales, stream)
        product(weights.down[layer], wide_codes, 2 * hidden, added)
    count = len(last_rows)
    x, added, logits = x[last_rows], added[last_rows], rows(len(model.embedding), torch.float32, count)
    hb.hfx_rms_norm(weights.norm, count, added, hidden, x, hidden, x, None, codes, scales, stream)
    hb.hfx_matmul_rows(weights.embedding, count, codes, hidden, scales, logits, logits.shape[1], True, stream)
    return logits


def serve(model, cache, prompts, new_tokens, forced=None, held=None, weights=None):
    """Serves the prompts (lists of token ids) until each has `new_tokens` tokens.  Returns their tokens, their logits and the steps' times in seconds.
    forced: tokens to go on with in place of the likeliest ones.  weights: the model's Weights8, to serve with those."""
    latency = hb.hfx_latency_model(1e-3, 2e-5, 2e-2)              # seconds: of a prefill batch, of each of its tokens, of a decode iteration
    waiting = list(range(len(prompts)))
    running, pages, length = [], {}, {}
    tokens = {r: [] for r in waiting}
    logits = {r: [] for r in waiting}
    times = []
    while waiting or running:
        started = time.perf_counter()
        admitted, kind, q_len, ctx_len, decision = hb.hfx_compose_step(0.2, 0.05, latency, [length[r] for r in running], [len(prompts[r]) for r in waiting],
                                                                       mixed=True)
        if not len(kind):
            raise RuntimeError("the longest prompt is over the token budget of a step (%d)" % decision.budget)
        chosen = [r for r, a in zip(waiting, admitted) if a]
        batch = running + chosen                                  # the order in which the step has them
        waiting = [r for r, a in zip(waiting, admitted) if not a]
        for r, n in zip(batch, ctx_len):
            length[r] = int(n)
            have = pages.setdefault(r, [])
            need = -(-length[r] // PAGE) - len(have)
            if need > len(cache.free):
                raise RuntimeError("out of pages")
            have += [cache.free.pop() for _ in range(need)]
        step = Step(cache, kind, q_len, ctx_len, [pages[r] for r in batch])
        packed = [t for r in batch for t in (tokens[r][-1:] if r in running else prompts[r])]
        packed, last_rows = torch.tensor(packed, device="cuda"), torch.from_numpy(np.cumsum(q_len) - 1).cuda()
        rows = forward_8(model, weights, cache, step, packed, last_rows) if weights else forward(model, cache, step, packed, last_rows, held)
        picked = rows.argmax(1).tolist()                          # (waits for the step)
        times.append(time.perf_counter() - started)
        for i, r in enumerate(batch):
            logits[r].append(rows[i])
            tokens[r].append(forced[r][len(tokens[r])] if forced else picked[i])
        running = []
        for r in batch:
            if len(tokens[r]) < new_tokens:
                running.append(r)
            else:
                cache.free += pages.pop(r)
    return tokens, {r: torch.stack(x) for r, x in logits.items()}, times


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--q-heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--head-dim", type=int, default=128, choices=(64, 128))
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--requests", type=int, default=24)
    ap.add_argument("--longest-prompt", type=int, default=1500)
    ap.add_argument("--new-tokens", type=int, default=32)
    ap.add_argument("--weights", type=int, default=16, choices=(16, 8), help="bits of the projections' weights and rows")
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    rng = np.random.default_rng(a.seed)
    vocab = 4096
    prompts = [rng.integers(0, vocab, rng.integers(1, a.longest_prompt + 1)).tolist() for _ in range(a.requests)]
    num_pages = sum(-(-(len(p) + a.new_tokens) // PAGE) for p in prompts)
    model = Decoder(a.q_heads, a.kv_heads, a.head_dim, a.layers, vocab, a.longest_prompt + a.new_tokens, a.seed)
    weights = Weights8(model) if a.weights == 8 else None
    served, held = {}, []
    for four_bits in (False, True):
        cache = Cache(model, num_pages, four_bits)
        forced = served[False][0] if four_bits else None
        tokens, logits, times = served[four_bits] = serve(model, cache, prompts, a.new_tokens, forced, held, weights)
        assert len(cache.free) == num_pages
        print("%-5s pool: %7.1f MB, %d steps, median %.2f ms a step" % (
            "4-bit" if four_bits else "bf16", sum(p.numel() for p in cache.pools) / 1e6, len(times), 1e3 * float(np.median(times))), flush=True)
    x, y = (torch.cat([served[f][1][r] for r in range(a.requests)]) for f in (False, True))
    off = float((x - y).norm() / x.norm())
    same = float((x.argmax(1) == y.argmax(1)).float().mean())
    print("logits over the 4-bit pool against those over the bf16 pool: %.3f off (relative), the same likeliest token in %.1f %% of %d%s" % (
        off, 100 * same, len(x), "; values in the pool %.3f off" % max(held) if held else ""))
    return {"off": off, "same": same, "values_off": max(held) if held else None, "tokens": {f: served[f][0] for f in served}}


if __name__ == "__main__":
    main()
