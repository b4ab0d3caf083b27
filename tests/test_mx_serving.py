"""The 4-bit cache in use: the serving example against a plain decoder, both pools on larger steps, pools past 4 GB, streams, captured graphs, steps of many runs.

Tolerances, from the arithmetic:
 * decoder: activations are rounded to bf16 about ten times a layer, 2^-9 of their size at most (0.0017 on average): 0.01 of the logits over two layers, of
   which 0.03 allow for what the layers make of it.  A rounding can also move a key or value to the next 4-bit code, and nothing averages that in a context of
   a few tokens; so the plain decoder takes keys and values as the 4-bit pool holds them, and those are bounded by the format: an element is off by at most a
   quarter of itself from one unit of its block's scale up, and by a quarter of a unit below; the largest element has 3.5 units at least, so in normal values
   the latter add less than 0.22 of the norm: (0.25^2 + 0.22^2)^0.5 = 0.333 in all.
 * the 4-bit pool against the bf16 pool that holds what it stands for: weights and results are rounded to bf16 on both sides (0.0017 each) and the queries
   by less, 0.0035 in all as a ratio of norms: 0.006.
 * everything else is the same arithmetic on the same numbers: equal bits.
"""
import importlib.util
import os

import numpy as np
import pytest

from tests.test_mx_cache import MAGNITUDES, Step, angles, attend, hb, random_pool  # noqa: F401  (hb is a fixture)

EXAMPLE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serving_loop.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("serving_loop", EXAMPLE)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def quantised(torch, x):
    """fp32 tensor [..., D] -> the values that the 4-bit format holds for it."""
    b = x.double().reshape(*x.shape[:-1], -1, 32)
    top = b.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top))
    size = torch.exp2(e - 2 + (top >= 1.75 * torch.exp2(e)))
    grid = torch.tensor(MAGNITUDES, dtype=torch.float64, device=x.device)
    y = (b / size).abs()
    middle = (grid[1:] + grid[:-1]) / 2
    code = (y[..., None] > middle).sum(-1) + (y[..., None] == middle)[..., 1::2].sum(-1)       # ties go to the even code
    return (grid[code] * b.sign() * size).reshape(x.shape)


HELD = (0.25 ** 2 + 0.22 ** 2) ** 0.5


def plain_logits(torch, model, tokens, held=None):
    """Logits after every token, by a plain decoder in 64 bits without a cache; held: keys and values [tokens, heads, d] of each layer to be taken for its own."""
    hq, hkv, d = model.hq, model.hkv, model.d
    n = len(tokens)
    position = torch.arange(n, device="cuda", dtype=torch.float64)
    angle = position[:, None] * 10000.0 ** (-torch.arange(d // 2, device="cuda", dtype=torch.float64) / (d // 2))
    c, s = angle.cos()[:, None], angle.sin()[:, None]

    def turn(x):
        a, b = x[..., :d // 2], x[..., d // 2:]
        return torch.cat((a * c - b * s, b * c + a * s), -1)

    def norm(x):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
    x = model.embedding.double()[torch.tensor(tokens, device="cuda")]
    hidden = torch.ones((n, n), device="cuda", dtype=torch.bool).triu(1)
    for layer in range(model.layers):
        qkv = norm(x) @ model.qkv[layer].double().T
        q, k, v = (y.reshape(n, -1, d) for y in qkv.split((hq * d, hkv * d, hkv * d), 1))
        q, k = turn(q), turn(k)
        if held:
            for own, taken in ((k, held[layer][0]), (v, held[layer][1])):
                assert float((taken - own).norm() / own.norm()) < HELD
            k, v = held[layer]
        rows = []
        for h in range(hq):
            w = (q[:, h] @ k[:, h // (hq // hkv)].T) / d ** 0.5
            rows.append(torch.softmax(w.masked_fill(hidden, -torch.inf), 1) @ v[:, h // (hq // hkv)])
        x = x + torch.stack(rows, 1).reshape(n, hq * d) @ model.out[layer].double().T
        y = norm(x) @ model.up[layer].double().T
        x = x + y * torch.sigmoid(y) @ model.down[layer].double().T
    return norm(x) @ model.embedding.double().T


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64)])
def test_the_serving_example_against_a_plain_decoder(hb, example, monkeypatch, hq, hkv, d):
    import torch
    new = 6
    g = np.random.default_rng(3)
    prompts = [g.integers(0, 300, n).tolist() for n in (1, 17, 130, 16, 75, 33)]
    model = example.Decoder(hq, hkv, d, 2, 300, 256, seed=4)
    num_pages = sum(-(-(len(p) + new) // 16) for p in prompts)
    steps = []

    class Recorded(example.Step):
        def __init__(self, cache, kind, q_len, ctx_len, pages):
            super().__init__(cache, kind, q_len, ctx_len, pages)
            steps.append((ctx_len.copy(), [list(p) for p in pages]))
    monkeypatch.setattr(example, "Step", Recorded)
    for four_bits in (False, True):
        cache = example.Cache(model, num_pages, four_bits)
        tokens, logits, times = example.serve(model, cache, prompts, new)
        assert len(cache.free) == num_pages and len(times) == new      # (all prompts in the first step, so no page has had a second owner)
        held = [None] * len(prompts)
        if four_bits:
            ctx, pages = steps[-1]
            assert ctx.tolist() == [len(p) + new - 1 for p in prompts]
            whole = example.Step(cache, np.ones(len(ctx), np.int32), ctx, ctx, pages)
            layers = []
            for pool in cache.pools:
                k, v = torch.empty((2, int(ctx.sum()), hkv, d), dtype=torch.bfloat16, device="cuda")
                hb.hfx_read_new_kv_mx(cache.shape, pool, whole.host, whole.device, k, v, torch.cuda.current_stream())
                layers.append((k.double().split(ctx.tolist()), v.double().split(ctx.tolist())))
            held = [[(k[r], v[r]) for k, v in layers] for r in range(len(prompts))]
        for r, p in enumerate(prompts):
            want = plain_logits(torch, model, p + tokens[r][:-1], held[r])[len(p) - 1:]
            off = float((logits[r].double() - want).norm() / want.norm())
            print(f"four bits {four_bits} request {r}: {off:.4f} off")
            assert off <= 0.03


@pytest.mark.gpu
def test_the_example_as_a_command(hb, example, capsys):
    got = example.main(["--q-heads", "4", "--kv-heads", "2", "--head-dim", "64", "--requests", "5", "--longest-prompt", "60", "--new-tokens", "5"])
    assert got["tokens"][True] == got["tokens"][False] and all(len(t) == 5 for t in got["tokens"][False].values())
    assert 0.02 < got["values_off"] < HELD
    assert "4-bit pool" in capsys.readouterr().out


def whole_contexts(hb, torch, step):
    """A descriptor under which all tokens of the step's contexts are new."""
    kind = np.ones(len(step.q_len), np.int32)
    n, _, _ = hb.hfx_batch_desc_sizes(step.shape, kind, step.ctx_len, step.ctx_len)
    host, dev = torch.empty(n, dtype=torch.uint8, pin_memory=True), torch.empty(n, dtype=torch.uint8, device="cuda")
    hb.hfx_build_batch_desc(step.shape, kind, step.ctx_len, step.ctx_len, step.indptr, step.pages, host, dev, torch.cuda.current_stream())
    return host, dev


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,q_len,ctx", [
    (32, 8, 128, [1] * 40 + [700, 129, 2], [1 + 220 * i for i in range(40)] + [5700, 129, 9000]),
    (8, 1, 128, [1, 1, 1, 1500], [30000, 17, 12345, 9000]),
    (64, 4, 128, [1] * 7 + [33], [70000, 1, 16, 900, 8000, 4097, 31, 4000]),
    (12, 4, 64, [1] * 30 + [400, 65], [64 * (i + 1) + i for i in range(30)] + [4400, 65]),
    (40, 8, 128, [3, 1, 31, 1], [20000, 20001, 33, 1]),
])
def test_both_pools_on_larger_steps(hb, hq, hkv, d, q_len, ctx):
    """Items split along the keys, merges, groups of 1 to 16 heads: the 4-bit pool against the bf16 pool that holds what it stands for."""
    import torch
    step = Step(hb, hq, hkv, d, q_len, ctx, 17)
    stream = torch.cuda.current_stream()
    gen = torch.Generator(device="cuda").manual_seed(5)
    mx = torch.randint(0, 256, (step.num_pages, hkv, 17 * d), dtype=torch.uint8, device="cuda", generator=gen)
    mx[:, :, 16 * d:] = mx[:, :, 16 * d:] % 3 + 124
    total = int(step.ctx_len.sum())
    k, v = torch.empty((2, total, hkv, d), dtype=torch.bfloat16, device="cuda")
    host, dev = whole_contexts(hb, torch, step)
    hb.hfx_read_new_kv_mx(step.shape, mx, host, dev, k, v, stream)
    pool = torch.zeros((step.num_pages, hkv, 2, 16 * d), dtype=torch.bfloat16, device="cuda")
    hb.hfx_append_kv(step.shape, k, v, pool, host, dev, stream)
    q = torch.empty((step.tokens, hq, d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    out = torch.full((2, step.tokens, hq, d), torch.nan, dtype=torch.bfloat16, device="cuda")
    hb.hfx_mixed_paged_attention(step.shape, q, pool, step.host, step.dev, step.ws, out[0], stream)
    hb.hfx_mixed_paged_attention_mx(step.shape, q, mx, step.host, step.dev, step.ws, out[1], stream)
    a, b = out.double()
    assert bool(torch.isfinite(out).all())
    off = float((a - b).norm() / a.norm())
    print(f"{off:.5f} off")
    assert off <= 0.006


def run_all(hb, torch, step, rows, rope, mx, q, out, k_out, v_out, stream):
    """The calls of a layer: rotation and append, the way back, attention."""
    hq, hkv, d = step.hq, step.hkv, step.d
    qs, ks, vs = rows.split((hq * d, hkv * d, hkv * d), 1)
    hb.hfx_rope_append_kv_mx(step.shape, rope, qs, qs.stride(0), ks, ks.stride(0), vs, vs.stride(0), q, mx, step.host, step.dev, stream)
    hb.hfx_read_new_kv_mx(step.shape, mx, step.host, step.dev, k_out, v_out, stream)
    hb.hfx_mixed_paged_attention_mx(step.shape, q, mx, step.host, step.dev, step.ws, out, stream)


def layer(hb, hq, hkv, d, q_len, ctx, seed, pool=None):
    """A step with its buffers: pool with earlier tokens, projected rows."""
    import torch
    step = Step(hb, hq, hkv, d, q_len, ctx, seed)
    mx = torch.from_numpy(random_pool(step)).cuda() if pool is None else pool
    rows = torch.empty((step.tokens, (hq + 2 * hkv) * d), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(seed))
    rope = hb.make_rope(torch.from_numpy(angles(int(max(ctx)), d)).cuda(), d)
    q, out = torch.empty((2, step.tokens, hq, d), dtype=torch.bfloat16, device="cuda")
    k_out, v_out = torch.empty((2, step.tokens, hkv, d), dtype=torch.bfloat16, device="cuda")
    return step, mx, rows, rope, q, out, k_out, v_out


@pytest.mark.gpu
def test_pools_past_4_gb(hb):
    """The same step on low page ids and on the last ones of pools whose offsets pass 32 bits: the same bits, in both pools."""
    import torch
    hq, hkv, d = 16, 8, 128
    q_len, ctx = [1, 1, 50], [100, 33, 200]
    step, mx, rows, rope, q, out, k_out, v_out = layer(hb, hq, hkv, d, q_len, ctx, 9)
    stream = torch.cuda.current_stream()
    mx0 = mx.clone()
    run_all(hb, torch, step, rows, rope, mx, q, out, k_out, v_out, stream)
    many = 260000                                             # 4.53e9 bytes in 4 bits
    assert many * hkv * 17 * d > 1 << 32
    far = Step(hb, hq, hkv, d, q_len, ctx, 9, extra=many - step.num_pages + 3)
    assert far.num_pages == many
    far.kind, far.pages = step.kind, (many - 1 - step.pages).astype(np.int32)
    hb.hfx_build_batch_desc(far.shape, far.kind, far.q_len, far.ctx_len, far.indptr, far.pages, far.host, far.dev, stream)
    big = torch.zeros((many, hkv, 17 * d), dtype=torch.uint8, device="cuda")
    big[many - step.num_pages:] = mx0.flip(0)
    q2, out2, k2, v2 = (torch.zeros_like(x) for x in (q, out, k_out, v_out))
    run_all(hb, torch, far, rows, rope, big, q2, out2, k2, v2, stream)
    torch.cuda.synchronize()
    for a, b in ((q, q2), (out, out2), (k_out, k2), (v_out, v2), (mx, big[many - step.num_pages:].flip(0))):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert not big[:many - step.num_pages].any()
    del big
    n = 70000                                                 # 4.59e9 bytes in bf16
    assert n * hkv * 2 * 16 * d * 2 > 1 << 32
    near = torch.zeros((step.num_pages, hkv, 2, 16 * d), dtype=torch.bfloat16, device="cuda")
    qs, ks, vs = rows.split((hq * d, hkv * d, hkv * d), 1)
    args = (rope, qs, qs.stride(0), ks, ks.stride(0), vs, vs.stride(0))
    hb.hfx_rope_append_kv(step.shape, *args, q, near, step.host, step.dev, stream)
    far = Step(hb, hq, hkv, d, q_len, ctx, 9, extra=n - step.num_pages + 3)
    far.kind, far.pages = step.kind, (n - 1 - step.pages).astype(np.int32)
    hb.hfx_build_batch_desc(far.shape, far.kind, far.q_len, far.ctx_len, far.indptr, far.pages, far.host, far.dev, stream)
    big = torch.zeros((n, hkv, 2, 16 * d), dtype=torch.bfloat16, device="cuda")
    hb.hfx_rope_append_kv(far.shape, *args, q2, big, far.host, far.dev, stream)
    torch.cuda.synchronize()
    assert torch.equal(q, q2) and torch.equal(near, big[n - step.num_pages:].flip(0)) and not big[:n - step.num_pages].any()


@pytest.mark.gpu
def test_another_stream(hb):
    import torch
    args = (8, 2, 128, [1, 40, 1], [500, 700, 90], 21)
    step, mx, rows, rope, q, out, k_out, v_out = layer(hb, *args)
    side = torch.cuda.Stream()
    mx2 = mx.clone()
    q2, out2, k2, v2 = (torch.zeros_like(x) for x in (q, out, k_out, v_out))
    run_all(hb, torch, step, rows, rope, mx, q, out, k_out, v_out, torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        run_all(hb, torch, step, rows, rope, mx2, q2, out2, k2, v2, side)
    side.synchronize()
    for a, b in ((mx, mx2), (q, q2), (out, out2), (k_out, k2), (v_out, v2)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,q_len,ctx", [(32, 8, 128, [1] * 6, [100, 2500, 33, 700, 1, 16]), (8, 2, 64, [1, 130, 33], [3000, 700, 33])])
def test_captured_calls(hb, hq, hkv, d, q_len, ctx):
    """A layer's calls in a graph: every replay gives what the calls give, on the inputs of that replay."""
    import torch
    step, mx, rows, rope, q, out, k_out, v_out = layer(hb, hq, hkv, d, q_len, ctx, 33)
    start = mx.clone()
    side = torch.cuda.Stream()
    run_all(hb, torch, step, rows, rope, mx, q, out, k_out, v_out, torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run_all(hb, torch, step, rows, rope, mx, q, out, k_out, v_out, side)
    for i in range(4):
        rows.normal_(generator=torch.Generator(device="cuda").manual_seed(50 + i))
        mx.copy_(start)
        for x in (q, out, k_out, v_out):
            x.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (mx, q, out, k_out, v_out)]
        mx.copy_(start)
        run_all(hb, torch, step, rows, rope, mx, q, out, k_out, v_out, torch.cuda.current_stream())
        torch.cuda.synchronize()
        for a, b in zip(got, (mx, q, out, k_out, v_out)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.gpu
def test_a_step_of_many_requests(hb):
    """More runs than one dimension of a grid takes, one new token each; and their attention, a context of one or two tokens."""
    import torch
    n, d = 40000, 64
    ctx = np.random.default_rng(2).integers(1, 3, n)
    step = Step(hb, 1, 1, d, [1] * n, ctx, 41)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v, q = (torch.empty((n, 1, d), dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(3))
    mx = torch.zeros((step.num_pages, 1, 17 * d), dtype=torch.uint8, device="cuda")      # scales of zero: earlier tokens' values are zero
    k_out, v_out, out = (torch.empty_like(k) for _ in range(3))
    stream = torch.cuda.current_stream()
    hb.hfx_rope_append_kv_mx(step.shape, None, None, 0, k, d, v, d, None, mx, step.host, step.dev, stream)
    hb.hfx_read_new_kv_mx(step.shape, mx, step.host, step.dev, k_out, v_out, stream)
    hb.hfx_mixed_paged_attention_mx(step.shape, q, mx, step.host, step.dev, step.ws, out, stream)
    torch.cuda.synchronize()
    kq, vq = quantised(torch, k), quantised(torch, v)
    assert torch.equal(k_out.double(), kq) and torch.equal(v_out.double(), vq)
    score = (q.double() * kq).sum(-1, keepdim=True) / d ** 0.5
    two = torch.from_numpy(ctx == 2).cuda()[:, None, None]
    want = vq * torch.where(two, torch.sigmoid(score), 1.0)                                # the earlier token has score and value zero
    err = (out.double() - want).abs()
    assert float(err.max()) <= 2e-2 and float(err.mean()) <= 2e-3


@pytest.mark.gpu
def test_values_that_are_not_finite_stay_in_their_request(hb):
    import torch
    step = Step(hb, 8, 2, 128, [1, 40, 1, 33], [300, 100, 50, 33], 61)
    pool = random_pool(step)
    q = step.bits(step.tokens, 8, 128)
    want = attend(step, q, torch.from_numpy(pool).cuda())
    bad = pool.copy()
    for r in (1, 2):
        bad[step.pages[step.indptr[r]], :, 16 * 128:] = 255      # the first page of the request stands for NaN
    got = attend(step, q, torch.from_numpy(bad).cuda())
    others = np.isin(step.request, (0, 3))
    assert np.array_equal(got[others], want[others]) and not np.array_equal(got[~others], want[~others])


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,interleaved", [(32, 8, 128, False), (32, 8, 128, True), (64, 16, 64, False), (64, 16, 64, True)])
def test_a_large_step_is_its_requests_one_by_one(hb, hq, hkv, d, interleaved):
    """Steps whose rows pass 64 MB take another way through the caches; each of the requests alone does not."""
    import torch
    q_len, ctx = [2001, 1, 1997], [2001, 77, 2500]
    step = Step(hb, hq, hkv, d, q_len, ctx, 71)
    g = torch.Generator(device="cuda").manual_seed(71)
    rows = torch.empty((step.tokens, (hq + 2 * hkv) * d), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    assert step.tokens * 2 * (hq + hkv) * d * 2 > 64 << 20 > 2001 * 2 * (hq + hkv) * d * 2
    rope = hb.make_rope(torch.from_numpy(angles(2500, d)).cuda(), d, interleaved)
    stream = torch.cuda.current_stream()

    def append(f, sizes, x, q, pool, host, dev):
        qs, ks, vs = x.split((hq * d, hkv * d, hkv * d), 1)
        f(sizes, rope, qs, qs.stride(0), ks, ks.stride(0), vs, vs.stride(0), q, pool, host, dev, stream)
    for f, shape, dtype in ((hb.hfx_rope_append_kv, (step.num_pages, hkv, 2, 16 * d), torch.bfloat16), (hb.hfx_rope_append_kv_mx, (step.num_pages, hkv, 17 * d), torch.uint8)):
        whole, parts = (torch.zeros(shape, dtype=dtype, device="cuda") for _ in range(2))
        q, q_parts = (torch.zeros((step.tokens, hq, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        append(f, step.shape, rows, q, whole, step.host, step.dev)
        kept, at = [], 0
        for r, n in enumerate(q_len):
            kind, one, c = step.kind[r:r + 1], step.q_len[r:r + 1], step.ctx_len[r:r + 1]
            size, _, _ = hb.hfx_batch_desc_sizes(step.shape, kind, one, c)
            host, dev = torch.empty(size, dtype=torch.uint8, pin_memory=True), torch.empty(size, dtype=torch.uint8, device="cuda")
            pages = step.pages[step.indptr[r]:step.indptr[r + 1]]
            hb.hfx_build_batch_desc(step.shape, kind, one, c, np.array([0, len(pages)], np.int32), pages, host, dev, stream)
            append(f, step.shape, rows[at:at + n], q_parts[at:at + n], parts, host, dev)
            kept.append((host, dev))
            at += n
        torch.cuda.synchronize()
        assert torch.equal(q.view(torch.int16), q_parts.view(torch.int16)) and torch.equal(whole.view(torch.uint8), parts.view(torch.uint8)) and bool(whole.any())


def test_which_steps_read_pages_past_the_caches():
    """Large steps, unless their requests share leading pages that the caches serve; planned on the host."""
    from paper_2508_15919_amd import binding
    hq, hkv, d = 32, 8, 128
    page = 17 * hkv * d

    def flag(requests, pages_each, shared, kind=0):
        own = pages_each - shared
        ids = np.concatenate([np.concatenate((np.arange(shared), shared + i * own + np.arange(own))) for i in range(requests)]).astype(np.int32)
        ctx, q = np.full(requests, 16 * pages_each, np.int32), np.ones(requests, np.int32)
        shape = binding.make_shape(hq, hkv, d, shared + requests * own)
        kinds = np.full(requests, kind, np.int32)
        host = np.zeros(binding.hfx_batch_desc_sizes(shape, kinds, q, ctx)[0], np.uint8)
        binding.hfx_fill_batch_desc(shape, kinds, q, ctx, (np.arange(requests + 1) * pages_each).astype(np.int32), ids, host)
        return binding.parse_desc(host)["header"].stream_mx
    many, behind = (64 << 20) // page + 1, (3 << 20) // page + 1
    assert flag(8, many // 8 + 1, 0) == 1 and flag(8, many // 8 - 8, 0) == 0 and flag(1, many, 0) == 1
    assert flag(8, many // 8 + 1, behind) == 0 and flag(8, many // 8 + 1, behind - 1) == 1
    assert flag(500, behind + 20, behind) == 0 and flag(500, behind + 20, 0) == 1


@pytest.mark.gpu
def test_both_pools_where_pages_go_past_the_caches(hb):
    test_both_pools_on_larger_steps(hb, 8, 8, 64, [1, 1, 1, 40], [60000, 70001, 50000, 900])
    test_both_pools_on_larger_steps(hb, 16, 8, 128, [1, 1, 33], [40000, 30001, 700])


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (16, 1, 128)])
@pytest.mark.parametrize("q_len,ctx", [([1], [1]), ([64], [64]), ([65], [65]), ([33], [191]), ([128], [128]), ([129], [193]), ([300], [300]), ([2], [777]),
                                       ([1, 31, 64], [64, 700, 65]), ([100], [2000]), ([32, 32], [1025, 63])])
def test_prompts_alone(hb, hq, hkv, d, q_len, ctx):
    """Steps without decodes and with few items: keys of one step, of an odd and of an even number of steps, behind earlier tokens, cut into splits or not."""
    from tests.test_mx_cache import MAX_ABS, MEAN_ABS, dense
    from paper_2508_15919_amd.synth import bf16_bits_to_f64
    import torch
    step = Step(hb, hq, hkv, d, q_len, ctx, 300 + len(q_len) + q_len[0])
    step.kind[:] = 1
    size, _, ws = hb.hfx_batch_desc_sizes(step.shape, step.kind, step.q_len, step.ctx_len)
    step.host, step.dev = torch.empty(size, dtype=torch.uint8, pin_memory=True), torch.empty(size, dtype=torch.uint8, device="cuda")
    step.ws = torch.empty(ws, dtype=torch.uint8, device="cuda") if ws else None
    hb.hfx_build_batch_desc(step.shape, step.kind, step.q_len, step.ctx_len, step.indptr, step.pages, step.host, step.dev, torch.cuda.current_stream())
    pool = random_pool(step)
    q = step.bits(step.tokens, hq, d)
    got = bf16_bits_to_f64(attend(step, q, torch.from_numpy(pool).cuda()))
    err = np.abs(got - dense(step, bf16_bits_to_f64(q), pool))
    assert np.isfinite(got).all() and err.max() <= MAX_ABS and err.mean() <= MEAN_ABS


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("kinds,q_len,ctx", [("decodes", [1, 1, 1], [1500, 333, 64]), ("mixed", [1, 70, 1, 33], [700, 500, 90, 33]), ("prompts", [90, 64], [900, 300]),
                                             ("prompts", [200], [200])])
def test_maxima_that_keep_growing(hb, hq, hkv, d, kinds, q_len, ctx):
    """Scores with a spread of a dozen and more, keys that get larger along the context: reference exponents are outgrown again and again, and most weights vanish.
    The queries are numbers of four significant bits and one size, so that scores are exact but for the order of their sums, and the usual bounds hold."""
    from tests.test_mx_cache import MAX_ABS, MEAN_ABS, dense, place_tables
    from paper_2508_15919_amd.synth import bf16_bits_to_f64, f32_to_bf16_bits
    import torch
    step = Step(hb, hq, hkv, d, q_len, ctx, 500 + len(q_len) + d, scale=0.6)
    step.kind[:] = [0 if n == 1 and kinds != "prompts" else 1 for n in q_len]
    size, _, ws = hb.hfx_batch_desc_sizes(step.shape, step.kind, step.q_len, step.ctx_len)
    step.host, step.dev = torch.empty(size, dtype=torch.uint8, pin_memory=True), torch.empty(size, dtype=torch.uint8, device="cuda")
    step.ws = torch.empty(ws, dtype=torch.uint8, device="cuda") if ws else None
    hb.hfx_build_batch_desc(step.shape, step.kind, step.q_len, step.ctx_len, step.indptr, step.pages, step.host, step.dev, torch.cuda.current_stream())
    pool = random_pool(step)
    scales = place_tables(d)[4]                                # [16 slots][blocks]: bytes of the key scales
    for r, c in enumerate(step.ctx_len.tolist()):
        for t in range(c):
            page, at = step.pages[step.indptr[r] + t // 16], scales[t % 16]
            pool[page][:, at] -= np.uint8(5 - 5 * (t + 1) // c)
    q = f32_to_bf16_bits(step.g.choice(np.array([-3.75, -2.5, -1.5, -1, 1, 1.25, 2, 3.5], np.float32), (step.tokens, hq, d)))
    got = bf16_bits_to_f64(attend(step, q, torch.from_numpy(pool).cuda()))
    err = np.abs(got - dense(step, bf16_bits_to_f64(q), pool))
    print(f"max-abs {err.max():.3e} mean-abs {err.mean():.3e}")
    assert np.isfinite(got).all() and err.max() <= MAX_ABS and err.mean() <= MEAN_ABS
