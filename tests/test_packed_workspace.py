"""Workspace of tboa_packed_linear and tboa_packed_swiglu as the library reports it (CPU: host arithmetic)."""
import ctypes

import pytest

import paper_2602_04929_amd as tb

MOST = 8192      # tokens of one round; more go round by round through one workspace
SHAPES = [(4096, 4096, 4, 128), (2048, 2048, 4, 128), (10240, 8192, 4, 128), (8192, 8192, 4, 128), (4096, 11008, 4, 128), (11008, 4096, 4, 128), (13824, 5120, 3, 128), (4096, 4096, 8, 0),
          (1003, 1024, 2, 64), (300, 320, 3, 32)]


def room(shape, tokens, dtype):
    return int(tb.binding._lib.tboa_packed_workspace_bytes(ctypes.byref(tb.binding.PackedWeightDesc(*shape, None, None, None)), tokens, dtype))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_no_round_needs_more_than_the_call(shape, dtype):
    """The last round of a call of more than 8192 tokens has fewer of them, and may need more."""
    for tokens in [MOST + n for n in (1, 65, 300, 1000, 2000, 2048, 3000, 4096, 5000, 6000, 7000, 8000)] + [2 * MOST, 2 * MOST + 2048, 1 << 24]:
        assert room(shape, tokens, dtype) >= max(room(shape, MOST, dtype), room(shape, tokens % MOST, dtype)), tokens


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_fewer_tokens_need_no_more(shape, dtype):
    """What is reserved for the largest batch does for every smaller one (bf16 calls of 33 to 64 tokens take the kernel for few, others that for many, both from one workspace)."""
    most = 0
    for tokens in sorted({*range(1, 300), *range(300, 2 * MOST, 97), *range(256, 2 * MOST, 256), *range(257, 2 * MOST, 256), 1 << 20, 1 << 24}):
        need = room(shape, tokens, dtype)
        assert need >= most, tokens
        most = need


@pytest.mark.parametrize("shape,many", [((300, 3 * 87381 * 16, 4, 87381 * 16), False), ((300, 8140704, 8, 208736), False), ((300, 1 << 20, 4, 1 << 19), True), ((300, 1 << 22, 4, 0), True), ((300, 1 << 21, 2, 1 << 14), True)])
def test_rows_whose_groups_are_found_by_a_product_of_32_bits(shape, many):
    """The kernel for many tokens, the only one of more than 64 that has a workspace, finds a channel's group by a reciprocal of 32 bits, exact while units of 16 channels times units of a group stay below 2^32."""
    d_out, d_in, bits, group = shape
    units = d_in // 16
    g = group // 16
    exact = g < 2 or all((x * ((2 ** 32 + g - 1) // g)) >> 32 == x // g for k in range(1, units // g + 1) for x in (k * g - 1, k * g))
    assert many == exact
    assert (room(shape, 1000, 0) > 0) == many      # (fp32: 64 tokens or fewer need none)
