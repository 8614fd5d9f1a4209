"""Which kernels of a sparse block's operators keep registers in scratch memory, as the comments beside them say: read from the built library's metadata."""
import re

import pytest

from paper_2601_21198_amd.build import LIB_PATH
from test_kernel_registers import kernels

NAME = re.compile(r"_GLOBAL__N_1\d+(zm_(?:norm|route|moe|layer)_[a-z_]*kernel)(.*)")


@pytest.fixture(scope="module")
def operators():
    found = []
    for k in kernels(LIB_PATH):
        m = NAME.search(k[".name"])
        if m:
            found.append((m.group(1), m.group(2), k))
    return found


def spilled(k):
    return k[".vgpr_spill_count"], k[".private_segment_fixed_size"]


def test_norm_router_and_tiles_use_none(operators):
    names = {n for n, _, _ in operators}
    assert {"zm_norm_kernel", "zm_route_tile_kernel", "zm_route_logits_kernel", "zm_route_choose_kernel", "zm_moe_list_kernel", "zm_moe_product_kernel", "zm_moe_wide_kernel",
            "zm_moe_join_kernel", "zm_moe_few_join_kernel", "zm_moe_widen_kernel", "zm_layer_middle_kernel", "zm_layer_join_kernel"} <= names
    for name, _, k in operators:
        if name not in ("zm_moe_few_first_kernel", "zm_moe_few_second_kernel", "zm_layer_product_kernel"):
            assert spilled(k) == (0, 0), k[".name"]


def test_calls_of_few_tokens_use_little(operators):
    seen = 0
    for name, _, k in operators:
        if name in ("zm_moe_few_first_kernel", "zm_moe_few_second_kernel"):
            seen += 1
            assert k[".vgpr_spill_count"] <= 8 and k[".private_segment_fixed_size"] <= 36, k[".name"]
    assert seen == 24


def test_products_of_one_and_two_vectors_use_none(operators):
    seen = 0
    for name, arguments, k in operators:
        if name == "zm_layer_product_kernel":
            long_codes, waves, vectors, rows, rest = (int(v) for v in re.match(r"ILb(\d)ELi(\d)ELi(\d)ELi(\d)ELb(\d)E", arguments).groups())
            seen += 1
            if vectors < 4 or (vectors == 4 and rows == 2):
                assert spilled(k) == (0, 0), k[".name"]
    assert seen == 32
