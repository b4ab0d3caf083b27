"""The serving example as a command: what it says of the two pools' logits.

Its second run goes on with the tokens of the first, so equal tokens say nothing of the pool.  The distance of the logits does where contexts are of a few tokens: there the attended
values are about half of a row's squares behind the first layer, and a pool that gave unrelated ones would put logits about 1 off (2^0.5 of half of the squares).  From
the format, keys and values are off by at most 0.333 of themselves, results by 0.47, behind two layers 0.47 x (2 x 0.5)^0.5: the bound is 0.5.  A row's own token keeps the
largest logit through that: hidden / 3^0.5 against hidden^0.5 times 3.6, the largest of 4096 normal numbers; hidden is 256.
"""
import pytest

from tests.test_mx_serving import example, hb  # noqa: F401  (fixtures)


@pytest.mark.gpu
@pytest.mark.parametrize("prompt", [1, 4])
def test_the_pools_logits_are_near_each_other(hb, example, prompt):  # noqa: F811
    got = example.main(["--q-heads", "4", "--kv-heads", "2", "--head-dim", "64", "--requests", "6", "--longest-prompt", str(prompt), "--new-tokens", "4"])
    print(f"{got['off']:.3f} off, {got['same']:.2f} the same")
    assert 0.005 < got["off"] <= 0.5
    assert got["same"] >= 0.9
