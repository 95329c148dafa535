"""Sizes and workspaces of the operators of a sequence at their edges, without a GPU."""
import random

import pytest

from paper_2607_11985_gb300 import binding as B

NONE = 2 ** 64 - 1


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2607_11985_gb300 import build
    build.build()


def test_step_workspace_of_nothing_and_of_too_much():
    """No tokens need none; rows beyond 31 bits are refused before anything is counted in them."""
    for batch, tokens in ((0, 1), (2, 0), (0, 0), (0, 1 << 29), (1 << 29, 0)):
        assert B.vqc_attention_step_workspace_bytes(batch, tokens, 4, 2, 8, 5000, 0, 0) == 0
    for sizes in ((1, 1 << 20, 65536, 1), (1, 1 << 16, 65536, 1), (1 << 15, 1, 65536, 65536), ((1 << 30) - 1, 1, 4, 1)):
        assert B.vqc_attention_step_workspace_bytes(*sizes, 64, 8192, 0, 0) == NONE
    assert B.vqc_attention_step_workspace_bytes(1, (1 << 16) - 1, 32768, 1, 64, 8192, 0, 0) < NONE


def test_workspaces_of_any_sizes():
    """Every size query answers, whatever the sizes."""
    rng = random.Random(1)
    ends = [0, 1, 2, 3, 7, 8, 16, 64, 65, 127, 128, 129, 1000, 4096, 65535, 65536, 65537, 1 << 20, (1 << 29) + 1, (1 << 30) - 1, 1 << 30, (1 << 31) - 1, 1 << 31, 1 << 40]
    size = lambda: rng.choice(ends) if rng.random() < 0.7 else int(2 ** rng.uniform(0, 31))
    for _ in range(20000):
        batch, tokens, groups, capacity, window, sinks = (size() for _ in range(6))
        heads, dim = groups * rng.choice((1, 2, 3, 64)) if rng.random() < 0.9 else size(), rng.choice((1, 8, 33, 64, 80, 128, 160, 256, 257))
        B.vqc_attention_step_workspace_bytes(batch, tokens, heads, groups, dim, capacity, window, sinks)
        B.vqc_norm_rotary_workspace_bytes(batch, tokens, heads, groups, dim)
        for dtype in (B.VQC_F32, B.VQC_BF16, B.VQC_F16):
            B.vqc_attention_workspace_bytes(rng.randrange(2), dtype, batch, tokens, heads, groups, dim, window, sinks, rng.randrange(2))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,groups", [(8, 8), (8, 2), (16, 1)])
def test_workspace_of_many_first_tokens(heads, groups, dim):
    """The backward's sums of pieces of queries are bounded, whatever stays visible: by those of 4 tiles of keys (two matrices of 128 rows
    of floats) for each of 152 SMs, beside two floats for each row of queries (in whole tiles) of every head."""
    pieces = 4 * 152 * 2 * 128 * dim * 4
    for batch, tokens, window, sinks in ((1, 32768, 4096, 16), (1, 32768, 128, 16000), (1, 131072, 1024, 4096), (1, 131072, 1024, 65000), (1, 262144, 1024, 65536),
                                         (4, 65536, 512, 300), (64, 8192, 64, 100), (1, 1 << 22, 1 << 12, 1 << 20)):
        for dtype in (B.VQC_BF16, B.VQC_F16):
            with_them, without = (B.vqc_attention_workspace_bytes(1, dtype, batch, tokens, heads, groups, dim, window, s, 1) for s in (sinks, 0))
            assert without <= 2 * 4 * batch * heads * tokens + 512
            assert with_them - without <= pieces, (batch, tokens, window, sinks)
    # few first tokens are cut as they were: one tile of each group, in pieces of the window and a tile
    one = B.vqc_attention_workspace_bytes(1, B.VQC_BF16, 1, 32768, heads, groups, dim, 4096, 16, 1) - B.vqc_attention_workspace_bytes(1, B.VQC_BF16, 1, 32768, heads, groups, dim, 4096, 0, 1)
    assert one == groups * (1 + -(-(32768 - 4096) // 4224)) * 2 * 128 * dim * 4
