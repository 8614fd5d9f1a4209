"""zm_route with more places than a wave has lanes, and with more tokens than one launch has threads for."""
import pytest
import torch

from paper_2601_21198_amd import zipmoe as zm
from test_gpu_route import check, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,hidden,experts,top_k", [(3, 256, 1024, 100), (40, 128, 200, 130), (5, 64, 70, 70), (2, 96, 1024, 1024), (600, 64, 128, 65), (64, 200, 256, 128)])
def test_many_places(tokens, hidden, experts, top_k):
    x, w = inputs(tokens, hidden, experts, "bf16")
    check(x, w, top_k)
    check(x, w, top_k, renormalise=True, scale=1.5)
    bias = torch.zeros(experts, device="cuda")
    bias[::3] = -float("inf")                                               # fewer experts than places in some of these
    check(x, w, top_k, bias=bias, renormalise=True)
