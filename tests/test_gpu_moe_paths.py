"""The kernels of zm_moe and zm_layer_moe that calls of few tokens take, each reached on purpose: tables of more than 64 pairs, two tiles of columns, products of
compressed experts in every width of vectors and rows.  Bounds are those of test_gpu_moe, with h in two bf16 parts: up to 32 tokens and 512 pairs."""
import math

import pytest
import torch

from paper_2601_21198_amd import zipmoe as zm
from test_gpu_moe import Case, layer_forward, layer_of

pytestmark = pytest.mark.gpu


def few(c):
    return c.tokens <= 32 and c.tokens * c.top_k <= 512


# ---- matrices as bf16: a table of pairs, one tile of columns (up to 16 tokens) and two ----

TABLES = [(16, 2048, 1024, 64, 8), (9, 136, 72, 12, 8), (12, 264, 136, 40, 8), (24, 200, 100, 9, 4), (32, 512, 384, 70, 8), (32, 200, 100, 2, 1), (31, 129, 65, 128, 16), (1, 64, 40, 128, 100),
          (4, 72, 24, 128, 128), (17, 1024, 256, 3, 3)]


@pytest.mark.parametrize("kind", ["bf16", "mx8"])
@pytest.mark.parametrize("tokens,hidden,inter,experts,top_k", TABLES)
def test_tables(tokens, hidden, inter, experts, top_k, kind):
    c = Case(tokens, hidden, inter, experts, top_k, kind, residual=tokens % 2 == 0)
    assert few(c) and (tokens > 16 or tokens * top_k > 64)
    got = c.forward()
    c.check(got, few=True)
    assert torch.equal(c.forward(), got)


@pytest.mark.parametrize("tokens,top_k", [(12, 8), (16, 5), (24, 4), (32, 3)])
def test_tables_of_some_experts(tokens, top_k):
    """named out of order and not all, pairs left out, a popular expert, matrices of those that nobody chose not read"""
    c = Case(tokens, 264, 136, 20, top_k, dropped=0.3, zipf=1.5, pad=5)
    c.check(c.forward(), few=True)
    names = [19, 3, 0, 11, 7, 1, 2]
    c.ids[c.ids == 7] = 5
    for m in c.w:
        m[7] = float("nan")
        m[12] = float("nan")
    c.check(c.forward(names), names, few=True)
    c.ids[:] = -1
    assert torch.equal(c.forward(names), c.residual)


@pytest.mark.parametrize("tokens,top_k", [(12, 8), (16, 6), (20, 3), (32, 4)])
def test_tables_of_one_expert_for_all(tokens, top_k):
    c = Case(tokens, 256, 96, 12, top_k)
    c.ids[:] = 4                                                            # every pair the same: a token names it top_k times
    c.check(c.forward(), few=True)
    c.ids[:, 1:] = -1
    c.check(c.forward(), few=True)
    c.ids[:, 1], c.ids[:, 2] = 9, 4
    c.check(c.forward(), few=True)


@pytest.mark.parametrize("tokens,top_k", [(12, 8), (32, 4)])
def test_tables_with_a_token_that_is_not_finite(tokens, top_k):
    c = Case(tokens, 96, 80, 12, top_k)
    clean = c.forward().clone()
    c.x[1, 7] = float("nan")
    got = c.forward()
    others = [t for t in range(tokens) if t != 1]
    assert torch.all(torch.isnan(got[1])) and torch.equal(got[others], clean[others])


@pytest.mark.parametrize("tokens,top_k", [(13, 8), (32, 4)])
def test_tables_in_a_graph(tokens, top_k):
    c = Case(tokens, 256, 96, 12, top_k)
    experts = zm.Experts(c.pointers(), c.names, 256, 96)
    ws, out = c.workspace(experts.workspace_bytes(tokens, top_k)), torch.empty(tokens, 256, dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        experts.forward(c.x, c.ids, c.weights, out, ws, residual=c.residual, stream=torch.cuda.current_stream().cuda_stream)
    for k in range(3):
        other = Case(tokens, 256, 96, 12, top_k, seed=k + 1)
        c.x.copy_(other.x), c.ids.copy_(other.ids), c.weights.copy_(other.weights)
        c.x64 = other.x64
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        c.check(out, few=True)


# ---- compressed experts, multiplied as they are decoded ----

def rows_of_a_stream(width, stream):
    return stream // width if stream % width == 0 else 1 if width % stream == 0 else stream // width + 2


def multiplied(c, stream):
    return (c.tokens <= 8 and c.tokens * c.top_k <= 64 and c.hidden % 8 == 0 and c.inter % 8 == 0 and stream <= 8192 and
            max(rows_of_a_stream(c.hidden, stream), rows_of_a_stream(c.inter, stream)) <= 4)


# hidden, inter, chunk, stream: one and two rows, four; rows that straddle streams; last streams that are cut off inside a tile; rows of several streams
WIDTHS = [(256, 512, 4096, 512), (128, 256, 4096, 512), (200, 176, 2048, 512), (352, 360, 4096, 1024), (1376, 1368, 4096, 4096), (1024, 520, 1024, 512), (1536, 512, 2048, 1024)]


def fill(c, values):
    """the matrices' exponents: as they are (short codes), of many sizes (long codes), without any order (chunks kept raw), one value"""
    gen = torch.Generator().manual_seed(c.hidden + c.inter)
    for m in c.w:
        if values == "long":
            m.mul_(torch.exp(torch.randn(m.shape, generator=gen) * 2 - 4).cuda())
        elif values == "raw":
            m.mul_(torch.exp2(torch.randint(-100, 0, m.shape, generator=gen).float()).cuda())
        elif values == "one":
            m.fill_(0.03125)


@pytest.mark.parametrize("values", ["short", "long", "raw", "one"])
@pytest.mark.parametrize("hidden,inter,chunk,stream", WIDTHS)
@pytest.mark.parametrize("tokens", [1, 2, 4, 7])
def test_products(tokens, hidden, inter, chunk, stream, values):
    c = Case(tokens, hidden, inter, 4, 3, "mx8" if tokens == 4 else "bf16", residual=tokens != 2)
    assert multiplied(c, stream)
    fill(c, values)
    layer = layer_of(c, chunk, stream, 8 if values == "short" else 12)
    got = layer_forward(c, layer, c.names)
    c.check(got, few=True)
    assert torch.equal(layer_forward(c, layer, c.names), got)


def test_products_of_long_streams():
    c = Case(3, 4096, 2736, 1, 1)
    assert multiplied(c, 8192)
    c.check(layer_forward(c, layer_of(c, 16384, 8192), c.names), few=True)


@pytest.mark.parametrize("tokens,experts", [(8, 9), (8, 50), (5, 45)])
def test_products_of_64_pairs_and_many_experts(tokens, experts):
    """more matrices than a launch takes, short and long codes among them"""
    c = Case(tokens, 256, 256, experts, 8, zipf=0.3)
    assert multiplied(c, 512)
    gen = torch.Generator().manual_seed(experts)
    for m in c.w:
        m[1::2] *= torch.exp(torch.randn(m[1::2].shape, generator=gen) * 2 - 4).cuda()
    layer = layer_of(c, 4096, 512, 12)
    c.check(layer_forward(c, layer, sorted(set(c.ids.reshape(-1).tolist()))), few=True)
    c.check(layer_forward(c, layer, c.names), few=True)                     # and those that nobody chose


@pytest.mark.parametrize("tokens", [1, 2, 3, 8])
def test_products_of_some_experts(tokens):
    c = Case(tokens, 256, 512, 9, 4, dropped=0.3, zipf=1.0, pad=3)
    assert multiplied(c, 512)
    names = [8, 1, 3, 0]
    c.ids[c.ids == 3] = 5                                                   # nobody wants 3; 5 is not named
    for m in c.w:
        m[3] = float("nan")
        m[5] = float("nan")
    layer = layer_of(c, 2048, 512)
    c.check(layer_forward(c, layer, names), names, few=True)
    c.ids[:, 1] = c.ids[:, 0] = 1                                           # twice, once with another between
    c.ids[:, 3] = 1
    c.check(layer_forward(c, layer, names), names, few=True)
    c.ids[:] = -1
    assert torch.equal(layer_forward(c, layer, names), c.residual)
    assert torch.equal(layer_forward(c, layer, []), c.residual)


@pytest.mark.parametrize("tokens", [2, 8])
def test_products_with_a_token_that_is_not_finite(tokens):
    c = Case(tokens, 256, 512, 4, 2)
    layer = layer_of(c, 2048, 512)
    clean = layer_forward(c, layer, c.names).clone()
    c.x[1, 7] = float("nan")
    got = layer_forward(c, layer, c.names)
    others = [t for t in range(tokens) if t != 1]
    assert torch.all(torch.isnan(got[1])) and torch.equal(got[others], clean[others])


@pytest.mark.parametrize("kind", ["bf16", "mx8"])
@pytest.mark.parametrize("tokens", [1, 2, 4, 8])
def test_products_in_a_graph(tokens, kind):
    c = Case(tokens, 256, 512, 5, 2, kind)
    layer = layer_of(c, 2048, 512)
    ws, out = c.workspace(layer.moe_workspace_bytes(5, tokens, 2, 256)), torch.empty(tokens, 256, dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.moe(c.names, c.x, c.ids, c.weights, out, ws, scales=c.scales, residual=c.residual, stream=torch.cuda.current_stream().cuda_stream)
    for k in range(3):
        other = Case(tokens, 256, 512, 5, 2, kind, seed=k + 1)
        c.x.copy_(other.x), c.ids.copy_(other.ids), c.weights.copy_(other.weights)
        if kind == "mx8":
            c.scales.copy_(other.scales)
        c.x64 = other.x64
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        c.check(out, few=True)
