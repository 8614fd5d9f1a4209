"""zm_route with more places than a wave has lanes, and with more tokens than one launch has threads for."""
import pytest
import torch

from paper_2601_21198_amd import zipmoe as zm
from test_gpu_route import check, inputs, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,hidden,experts,top_k", [(3, 256, 1024, 100), (40, 128, 200, 130), (5, 64, 70, 70), (2, 96, 1024, 1024), (600, 64, 128, 65), (64, 200, 256, 128)])
def test_many_places(tokens, hidden, experts, top_k):
    x, w = inputs(tokens, hidden, experts, "bf16")
    check(x, w, top_k)
    check(x, w, top_k, renormalise=True, scale=1.5)
    bias = torch.zeros(experts, device="cuda")
    bias[::3] = -float("inf")                                               # fewer experts than places in some of these
    check(x, w, top_k, bias=bias, renormalise=True)


def test_more_tokens_than_a_launch_has_threads_for():
    """a tile of 16 tokens takes 1024 threads, and a launch has less than 2^32"""
    tokens, hidden, experts, top_k = (1 << 26) + 37, 8, 8, 2
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(tokens, hidden, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    w = torch.empty(experts, hidden, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    mask = (torch.arange(tokens, device="cuda") % 5 != 0).to(torch.uint8)
    ids = torch.full((tokens, top_k), -77, dtype=torch.int32, device="cuda")
    weights = torch.full((tokens, top_k), 77.0, device="cuda")
    ws = torch.empty(zm.route_workspace_bytes(tokens, hidden, experts), dtype=torch.uint8, device="cuda")
    zm.route(x, w, ids, weights, ws, token_mask=mask, renormalise=True)
    torch.cuda.synchronize()
    assert torch.all((ids >= -1) & (ids < experts)) and torch.equal(ids[:, 0] >= 0, mask != 0)
    for at in (0, (1 << 25) - 300, (1 << 26) - 300, tokens - 300):
        rows = slice(at, min(at + 600, tokens))
        want_ids, want_weights, _ = reference(x[rows], w, top_k, mask=mask[rows], renormalise=True)
        assert torch.equal(ids[rows].cpu(), want_ids)
        # differences of logits below 64, rounded to 32 bits, and sixteen more roundings
        assert torch.all((weights[rows].cpu().double() - want_weights).abs() <= (64 + 16) * 2.0 ** -23 * want_weights + 1e-37)
