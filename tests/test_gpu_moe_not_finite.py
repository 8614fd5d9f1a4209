"""What zm_moe and zm_layer_moe make of weights and scales that are not finite: what the formula gives, in calls of any number of tokens and from compressed
experts too."""
import math

import pytest
import torch

from test_gpu_moe import Case, layer_forward
from test_gpu_moe_paths import layer_of, reaches

pytestmark = pytest.mark.gpu
# tokens, top_k, compressed: one token, a lane per pair, a table of pairs, two tiles of columns, many tokens, large tiles; products while decoding, decoded first
CALLS = [(1, 2, False), (6, 2, False), (12, 8, False), (32, 4, False), (130, 2, False), (1500, 2, False), (1, 2, True), (2, 2, True), (4, 2, True), (8, 3, True), (40, 2, True)]


def case(tokens, top_k, compressed, kind="bf16"):
    """experts 3 and 6 have a token each at least"""
    c = Case(tokens, *((1024, 2048) if compressed and tokens == 8 else (256, 256)), 9, top_k, kind)
    c.ids[0, :2] = torch.tensor([3, 6], dtype=torch.int32)
    return c


def call(c, compressed):
    if not compressed:
        return c.forward()
    layer = layer_of(c, *((16384, 4096) if c.tokens == 8 else (2048, 1024)))
    assert reaches(c, layer, c.names) == (c.tokens <= 8)
    return layer_forward(c, layer, c.names)


@pytest.mark.parametrize("tokens,top_k,compressed", CALLS)
def test_infinite_weights_of_down(tokens, top_k, compressed):
    """an output of an expert's tokens is infinite, by the sign that h has"""
    c = case(tokens, top_k, compressed)
    c.w[2][3, 5, 40] = math.inf
    c.w[2][6, 7, 41] = -math.inf
    got = call(c, compressed).double()
    want, bound = c.exact(few=False)
    infinite = torch.isinf(want)
    assert torch.any(infinite) and not torch.any(torch.isnan(want))
    assert torch.equal(got[infinite], want[infinite])
    assert torch.all(((got - want).abs() <= bound)[~infinite])


@pytest.mark.parametrize("tokens,top_k,compressed", CALLS)
def test_one_significant_bit_meets_infinity(tokens, top_k, compressed):
    """h is a power of two: nothing is left of it behind its first bf16 part"""
    c = case(tokens, top_k, compressed)
    c.x.fill_(0)
    c.x[:, 0] = 1.0
    c.w[0][:, :, 0] = 128.0                     # silu(128) is 128: exp(-128) is below half a step of 1
    c.w[1][:, :, 0] = 0.5
    c.weights.fill_(0.25)
    c.w[2][3, 5, 40] = math.inf
    c.w[2][3, 9, 40] = -math.inf
    got = call(c, compressed)
    mine = (c.ids == 3).any(1)
    assert torch.all(got[mine][:, 5] == math.inf) and torch.all(got[mine][:, 9] == -math.inf)
    assert torch.all(torch.isfinite(got[~mine])) and torch.all(torch.isfinite(got[:, 10:]))


@pytest.mark.parametrize("tokens,top_k,compressed", CALLS)
def test_a_scale_that_is_not_a_number(tokens, top_k, compressed):
    """e8m0's 255, over zeros too"""
    c = case(tokens, top_k, compressed, "mx8")
    clean = call(c, compressed).clone()
    bad = sorted({0, tokens - 1})
    for t in bad:
        c.scales[t, 2] = 255
        c.x[t, 64:96] = torch.zeros(32, device="cuda").to(torch.float8_e4m3fn)
    got = call(c, compressed)
    assert torch.all(torch.isnan(c.scales.view(torch.float8_e8m0fnu).float()[bad, 2]))
    others = [t for t in range(tokens) if t not in bad]
    assert torch.all(torch.isnan(got[bad])) and torch.equal(got[others], clean[others])
