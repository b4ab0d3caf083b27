"""What the operators between a layer's attention steps are measured on: the norm of the residual stream, rows in 8 bits, and their products with
weights in 8 bits.

A case is a dict of plain values:
  entry      "norm":        residual plus x, root-mean-square norm of the sum, rows in bf16
             "norm_matmul": the same with the rows in 8 bits, and their product with a weight (projection to queries, keys and values; logits)
             "rows_matmul": rows to 8 bits, product (projection behind the attention)
             "silu_matmul": silu(gate) * up of a projection's rows to 8 bits, product (the end of a gated feed-forward)
             "matmul":      product of rows that are in 8 bits already (its beginning, behind the norm)
  rows       tokens of the step
  k, n       values of a row, and of a result's row
  bias, fp32 whether the product adds a bias, and whether results are fp32 (else bf16)
  gated      of "silu_matmul": rows are gate and up side by side; else silu of the rows alone

Rows in 8 bits: v_i stands as code_i * scale, scale = top / 127, top the largest |v_i|, codes whole numbers in [-127, 127], nearest, ties to even.  Weights are
held so by output channel.
"""
import math

import torch

own = False

EPS = 1e-6
# (k, n) of the drawn products: layers of 32 / 8 and of 64 / 8 heads of 128 and of 32 / 4 heads of 64, whole and as shares of one
PROJECTIONS = {
    "norm_matmul": ((4096, 6144), (4096, 16384), (8192, 1280), (2048, 2560), (1024, 1536), (2048, 32001), (4096, 4099), (5120, 7168)),
    "rows_matmul": ((4096, 4096), (1024, 8192), (2048, 2048), (512, 4096), (5120, 5120), (640, 2000)),
    "silu_matmul": ((8192, 4096), (2048, 8192), (4096, 2048), (1792, 4096), (10240, 5120), (1376, 1024)),
    "matmul": ((4096, 16384), (4096, 4096), (8192, 2048), (2048, 8192), (5120, 2560), (1040, 777), (16384, 4096)),
}
LARGEST = 2 * 4128 * 4096 * 16384


def _case(entry, rows, k, n=0, bias=False, fp32=False, gated=False, name=None):
    c = dict(entry=entry, rows=rows, k=k, n=n, bias=bias, fp32=fp32, gated=gated)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the last norm of a step with four decodes: a launch is all that counts
        _case("norm", 4, 4096, name="norm_few"),
        # the same of a step with long prompt chunks: bound by memory
        _case("norm", 8224, 4096, name="norm_chunks"),
        # the entrance of a layer's attention, four decodes: the weight's bytes, and two launches
        _case("norm_matmul", 4, 4096, 6144, name="qkv_few"),
        # ... of a large decode batch: bytes and matrix cores are about even
        _case("norm_matmul", 256, 4096, 6144, name="qkv_decodes"),
        # ... of a step with long prompt chunks: bound by the matrix cores
        _case("norm_matmul", 8224, 4096, 6144, name="qkv_chunks"),
        # a tensor-parallel share of a large layer (8 / 1 heads of 128 of 64 / 8), an odd batch, with a bias: few columns, long sums
        _case("norm_matmul", 37, 8192, 1280, bias=True, name="qkv_share"),
        # the projection behind that share's attention for one odd prompt: short sums
        _case("rows_matmul", 777, 1024, 8192, name="out_share"),
        # gate and up of a feed-forward for a batch of decodes: bound by the weight's bytes
        _case("matmul", 64, 4096, 16384, name="up_batch"),
        # the same for prompt chunks: the largest product of a layer
        _case("matmul", 4128, 4096, 16384, name="up_chunks"),
        # the end of that feed-forward, decodes
        _case("silu_matmul", 64, 8192, 4096, gated=True, name="down_batch"),
        # ... and an odd number of prompt tokens
        _case("silu_matmul", 2500, 8192, 4096, gated=True, name="down_chunks"),
        # logits in fp32 for the rows that are sampled, over a vocabulary of odd size
        _case("norm_matmul", 33, 2048, 32001, fp32=True, name="logits"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    entry = rng.choice(("norm", "norm_matmul", "norm_matmul", "rows_matmul", "silu_matmul", "matmul", "matmul"))
    if entry == "norm":
        return _case(entry, _log_int(rng, 1, 8224), rng.choice((512, 1024, 2048, 4096, 5120, 8192)))
    k, n = rng.choice(PROJECTIONS[entry])
    rows = _log_int(rng, 1, min(8224, LARGEST // (2 * k * n)))
    return _case(entry, rows, k, n, rng.random() < 0.25, entry in ("norm_matmul", "matmul") and rng.random() < 0.2, entry == "silu_matmul" and rng.random() < 0.7)


# ---------------------------------------------------------------- inputs
def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    entry, rows, k, n = (case[x] for x in ("entry", "rows", "k", "n"))

    def normal(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen)

    def codes(*shape):
        return normal(*shape).mul_(33.0).round_().clamp_(-127.0, 127.0).to(torch.int8)
    s = {"case": case}
    if entry.startswith("norm"):
        s["x"], s["residual"] = normal(rows, k), normal(rows, k)
        s["residual"] *= 3.0
        s["residual"][:, 5::97] *= 8.0              # channels that stand out of the residual stream
        s["gain"] = (1.0 + 0.2 * normal(k, dtype=torch.float32)).to(torch.bfloat16)
    elif entry == "rows_matmul":
        s["x"] = normal(rows, k)
    elif entry == "silu_matmul":
        both = normal(rows, 2 * k if case["gated"] else k)
        s["x"], s["times"] = both[:, :k], both[:, k:] if case["gated"] else None
    else:
        s["codes"] = codes(rows, k)
        s["scales"] = torch.exp(0.3 * normal(rows, dtype=torch.float32)) / 33.0
    if n:
        s["weight"] = codes(n, k)
        s["weight_scales"] = torch.exp(0.3 * normal(n, dtype=torch.float32)) / (33.0 * k ** 0.5)
        s["bias"] = normal(n) if case["bias"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    # what a program keeps for every step: the handles of its weights, and the rows that pass between calls
    from paper_2508_15919_amd import binding as hb
    s["hb"], rows, k, n = hb, case["rows"], case["k"], case["n"]
    if case["entry"].startswith("norm"):
        s["norm"] = hb.make_norm(s["gain"], EPS)
        s["sum"] = torch.empty_like(s["x"])
    if n:
        s["handle"] = hb.make_weight_q8(s["weight"], s["weight_scales"], s["bias"])
        s["out"] = torch.empty((rows, n), dtype=torch.float32 if case["fp32"] else torch.bfloat16, device="cuda")
        if case["entry"] != "matmul":
            s["codes"] = torch.empty((rows, k), dtype=torch.int8, device="cuda")
            s["scales"] = torch.empty(rows, dtype=torch.float32, device="cuda")
    else:
        s["out"] = torch.empty_like(s["x"])
    return s


# ---------------------------------------------------------------- one pass
def _plain_rows(v):
    """fp32 rows -> codes and the largest magnitude of each row, in fp32."""
    top = v.abs().amax(1, keepdim=True).clamp_min(2.0 ** -100)
    return torch.round(v * (torch.full_like(top, 127.0) / top)), top


def _plain(s):
    case = s["case"]
    entry = case["entry"]
    outs = ()
    if entry.startswith("norm"):
        h = (s["x"].float() + s["residual"].float()).to(torch.bfloat16)
        outs = (h,)
        h = h.float()
        r = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
        if entry == "norm":
            return h.to(torch.bfloat16), (h * r * s["gain"].float()).to(torch.bfloat16)
        codes, top = _plain_rows(h * s["gain"].float())
        scales = top * r / 127.0
    elif entry == "matmul":
        codes, scales = s["codes"].float(), s["scales"][:, None]
    else:
        v = s["x"].float()
        if entry == "silu_matmul":
            v = v / (1.0 + torch.exp(-v))
            if s["times"] is not None:
                v = v * s["times"].float()
        codes, top = _plain_rows(v)
        scales = top / 127.0
    y = (codes @ s["weight"].float().T) * scales * s["weight_scales"]
    if s["bias"] is not None:
        y += s["bias"].float()
    return (*outs, y if case["fp32"] else y.to(torch.bfloat16))


def run(s):
    if not own:
        return _plain(s)
    hb, case, stream = s["hb"], s["case"], torch.cuda.current_stream()
    entry, rows, k = case["entry"], case["rows"], case["k"]
    if entry == "norm":
        hb.hfx_rms_norm(s["norm"], rows, s["x"], k, s["residual"], k, s["sum"], s["out"], None, None, stream)
        return s["sum"], s["out"]
    if entry == "norm_matmul":
        hb.hfx_rms_norm(s["norm"], rows, s["x"], k, s["residual"], k, s["sum"], None, s["codes"], s["scales"], stream)
    elif entry != "matmul":
        x, times = s["x"], s.get("times")
        hb.hfx_quantise_rows(hb.HFX_ACT_SILU if entry == "silu_matmul" else hb.HFX_ACT_NONE, rows, k, x, x.stride(0), times,
                             0 if times is None else times.stride(0), None, s["codes"], s["scales"], stream)
    hb.hfx_matmul_rows(s["handle"], rows, s["codes"], k, s["scales"], s["out"], case["n"], case["fp32"], stream)
    return (s["sum"], s["out"]) if entry == "norm_matmul" else (s["out"],)


def work(case):
    entry, rows, k, n = (case[x] for x in ("entry", "rows", "k", "n"))
    nbytes = n * k + 4 * n + (2 * n if case["bias"] else 0) + rows * n * (4 if case["fp32"] else 2)
    flops = 2 * rows * n * k
    if entry == "norm":
        return {"bytes": 8 * rows * k + 2 * k, "flops": 5 * rows * k}
    if entry == "norm_matmul":
        return {"bytes": nbytes + 6 * rows * k + 2 * k, "flops": flops + 7 * rows * k}
    if entry == "matmul":
        return {"bytes": nbytes + rows * k + 4 * rows, "flops": flops}
    return {"bytes": nbytes + rows * k * (4 if case["gated"] and entry == "silu_matmul" else 2), "flops": flops + 3 * rows * k}


# ---------------------------------------------------------------- in 64 bits, from the definition
def _exact_codes(v, steps):
    """Codes and scales of rows in 64 bits.  steps: as the operator goes on from values that are given exactly, with the factor 127 / top and the products rounded
    to 32 bits, for next to a tie those decide."""
    top = v.abs().max(1, keepdim=True).values.clamp_min(2.0 ** -100)
    if not steps:
        return torch.round(v * 127.0 / top), top / 127.0
    factor = (127.0 / top).float().double()
    return torch.round((v * factor).float().double()), top / 127.0


def exact(case, seed):
    s = _inputs(case, seed)
    entry = case["entry"]
    outs = []
    if entry.startswith("norm"):
        total = s["x"].double() + s["residual"].double()
        outs.append(total)
        h = total.to(torch.bfloat16).double()                          # the norm is that of the stream as it is kept
        size = (h.pow(2).sum(1, keepdim=True) / case["k"] + EPS).sqrt()
        if entry == "norm":
            return total, h / size * s["gain"].double()
        codes, scales = _exact_codes(h * s["gain"].double(), True)
        scales = scales / size
    elif entry == "matmul":
        codes, scales = s["codes"].double(), s["scales"].double().unsqueeze(1)
    else:
        v = s["x"].double()
        if entry == "silu_matmul":
            v = v * torch.sigmoid(v)
            if s["times"] is not None:
                v *= s["times"].double()
        codes, scales = _exact_codes(v, entry == "rows_matmul")
    y = torch.mm(codes, s["weight"].double().t())
    y *= scales
    y *= s["weight_scales"].double()
    if s["bias"] is not None:
        y += s["bias"].double()
    return (*outs, y)
