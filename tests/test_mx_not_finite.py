"""The rotating appends where the projection's output holds infinities, NaN and the largest numbers: the operators' words about such values hold through the rotation.

Oracle and roundings are those of test_mx_cache: bits are equal, NaN stands where the oracle's arithmetic has one, and a block of 32 with a value that is not finite has the scale byte 255.
"""
import subprocess

import numpy as np
import pytest

from paper_2508_15919_amd import build
from paper_2508_15919_amd.synth import bf16_bits_to_f64, f32_to_bf16_bits
from tests.test_mx_cache import Step, angles, down, hb, place_tables, quantise, rotate  # noqa: F401  (hb is a fixture)


def test_the_append_is_compiled_for_values_that_are_not_finite(monkeypatch):
    """Its arithmetic takes what a projection wrote: under -fno-honor-nans a NaN there has no defined effect, least of all on what is tested about it afterwards."""
    ran = []

    class Compiler:
        returncode, stderr, stdout = 0, "", ""

        def __init__(self, command, **_):
            ran.append(command)

        def communicate(self, *_, **__):
            return "", ""

        def wait(self, *_, **__):
            return 0
        __enter__ = lambda self: self                # noqa: E731
        __exit__ = lambda self, *_: None             # noqa: E731
    monkeypatch.setattr(subprocess, "Popen", Compiler)
    monkeypatch.setattr(subprocess, "run", Compiler)
    build.build()
    compiled = [c for c in ran if any(str(a).endswith("hfx_append.hip") for a in c)]
    assert len(compiled) == 1
    assert not {"-fno-honor-nans", "-ffast-math", "-ffinite-math-only"} & set(compiled[0])
    packed = [c for c in ran if any(str(a).endswith(".hip") for a in c)]
    assert all("-packed-fp32-ops" in c and "--offload-arch=gfx950" in c for c in packed)


def special(step, heads):
    """Rows with all kinds of values that arithmetic trips over, in either half of a head and either place of a pair."""
    bits = step.bits(step.tokens, heads, step.d)
    flat = bits.reshape(-1, step.d)
    kinds = [0x7F80, 0xFF80, 0x7FC0, 0xFFFF, 0x7F7F, 0xFF7F, 0x0001, 0x8000]
    for i in range(0, len(flat), 3):                                  # two rows of three stay as they are
        flat[i, step.g.integers(0, step.d, 2)] = step.g.choice(kinds, 2)
    flat[1] = 0x7F7F                                                  # whose products and sums overflow
    return bits


def same(got, want, what):
    """Bits, but for which NaN it is."""
    g, w = bf16_bits_to_f64(got), bf16_bits_to_f64(want)
    assert np.array_equal(np.isnan(g), np.isnan(w)), what
    assert np.array_equal(np.where(np.isnan(g), 0, got), np.where(np.isnan(w), 0, want)), what


@pytest.mark.gpu
@pytest.mark.parametrize("q_len,ctx", [([1] * 9 + [2, 5], [3 + 7 * i for i in range(9)] + [2, 40]), ([40, 17, 1], [90, 17, 5])])
@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("rot,interleaved", [(128, False), (128, True), (64, False), (48, True)])
@pytest.mark.parametrize("d", [64, 128])
def test_rotated_values_that_are_not_finite(hb, d, rot, interleaved, four, q_len, ctx):
    rot = min(rot, d)
    hq, hkv = 8, 4
    step = Step(hb, hq, hkv, d, q_len, ctx, 500 + rot)
    torch, stream = step.torch, step.torch.cuda.current_stream()
    q, k, v = special(step, hq), special(step, hkv), special(step, hkv)
    table = angles(int(max(ctx)), rot)
    rope = hb.make_rope(torch.from_numpy(table).cuda(), rot, interleaved)
    out = torch.zeros((step.tokens, hq, d), dtype=torch.int16, device="cuda")
    size = (step.num_pages, hkv, 17 * d) if four else (step.num_pages, hkv, 2, 16 * d)
    dev = torch.zeros(size, dtype=torch.uint8 if four else torch.int16, device="cuda")
    append = hb.hfx_rope_append_kv_mx if four else hb.hfx_rope_append_kv
    append(step.shape, rope, step.up(q), hq * d, step.up(k), hkv * d, step.up(v), hkv * d, out, dev, step.host, step.dev, stream)
    torch.cuda.synchronize()

    def turned(x):
        with np.errstate(all="ignore"):
            return rotate(bf16_bits_to_f64(x), step.position, table, rot, interleaved, True)
    with np.errstate(all="ignore"):
        same(down(out), f32_to_bf16_bits(turned(q).astype(np.float32)), "queries")
        kr = turned(k)
        assert not np.isfinite(kr).all()
        if four:
            kb, ks, vb, vs, ke, ve = place_tables(d)
            pool = dev.cpu().numpy()
            for t in range(step.tokens):
                block, slot = pool[step.page[t]], step.slot[t]
                for x, byte, shift, scale, what in ((kr[t], kb, ks, ke, "keys"), (bf16_bits_to_f64(v[t]), vb, vs, ve, "values")):
                    code, e = quantise(x)
                    assert np.array_equal(block[:, scale[slot]], e), (what, t)
                    held = np.repeat(e != 255, 32, axis=-1)           # (codes of a block of NaN may be any)
                    assert np.array_equal(((block[:, byte[slot]] >> shift[slot]) & 15)[held], code[held]), (what, t)
        else:
            keys = f32_to_bf16_bits(kr.astype(np.float32))
            pool = down(dev)
            pk, pv = pool.reshape(step.num_pages, hkv, 2, d // 16, 16, 16), pool.reshape(step.num_pages, hkv, 2, d, 16)
            for t in range(step.tokens):
                same(pk[step.page[t], :, 0, :, step.slot[t]].reshape(hkv, d), keys[t], ("keys", t))
                assert np.array_equal(pv[step.page[t], :, 1, :, step.slot[t]], v[t]), ("values", t)
