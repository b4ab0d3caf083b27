"""The serving example with its projections in 8 bits, against a plain decoder in 64 bits that has the weights as they are held.

Tolerance, from the arithmetic: a row that is held in 8 bits is off by top / 127 / 12^0.5 of a value (a uniform error of one step) and top is about four times the size of the values, six of
those behind silu: 0.010 and 0.015 of the row.  Queries, keys and values are off by 0.010, scores of order 1 by 2^0.5 of that, attended rows by 0.018 in all, 0.021 behind the next rounding to 8 bits; the
feed-forward's part by 0.010 and 0.015, 0.02 in all with the activation's slope.  Either is a part of the row to which it is added; over two layers, what earlier ones were off going
through the later ones: less than 0.05, and bf16's roundings, ten a layer of 0.0017, 0.01.
"""
import numpy as np
import pytest

from tests.test_mx_serving import example, hb, plain_logits  # noqa: F401  (fixtures)


def held_weights(torch, handle):
    codes, scales, _ = handle.tensors
    return codes.double() * scales.double()[:, None]


class Held:
    """The decoder that plain_logits reads, with the weights that the 8-bit one has.  (The embedding's rows are looked up in bf16 and multiplied in 8 bits.)"""

    def __init__(self, torch, model, weights):
        self.hq, self.hkv, self.d, self.layers, self.embedding = model.hq, model.hkv, model.d, model.layers, model.embedding
        for name in ("qkv", "out", "up", "down"):
            setattr(self, name, [held_weights(torch, h) for h in getattr(weights, name)])


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64)])
def test_the_example_with_weights_in_8_bits(hb, example, hq, hkv, d):  # noqa: F811
    import torch
    new = 5
    g = np.random.default_rng(11)
    prompts = [g.integers(0, 300, n).tolist() for n in (1, 17, 130, 16, 75, 33)]
    model = example.Decoder(hq, hkv, d, 2, 300, 256, seed=6)
    weights = example.Weights8(model)
    num_pages = sum(-(-(len(p) + new) // 16) for p in prompts)
    cache = example.Cache(model, num_pages, False)
    tokens, logits, times = example.serve(model, cache, prompts, new, weights=weights)
    assert len(cache.free) == num_pages and len(times) == new
    plain = Held(torch, model, weights)
    # plain_logits multiplies with the embedding in bf16; the 8-bit one is off by 0.010 of a row, as above
    for r, p in enumerate(prompts):
        want = plain_logits(torch, plain, p + tokens[r][:-1])[len(p) - 1:]
        off = float((logits[r].double() - want).norm() / want.norm())
        print(f"request {r}: {off:.4f} off")
        assert 0.003 < off <= 0.06


@pytest.mark.gpu
def test_the_example_as_a_command_with_weights_in_8_bits(hb, example, capsys):  # noqa: F811
    got = example.main(["--q-heads", "4", "--kv-heads", "2", "--head-dim", "64", "--requests", "5", "--longest-prompt", "60", "--new-tokens", "5", "--weights", "8"])
    assert got["tokens"][True] == got["tokens"][False] and all(len(t) == 5 for t in got["tokens"][False].values())
    assert got["values_off"] is None and 0.0 < got["off"] <= 0.5
    assert "4-bit pool" in capsys.readouterr().out
