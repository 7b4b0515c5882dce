"""int2kv_token_weights_workspace_bytes of whole prompts: bounded, not growing with the square of their length (CPU only)."""
import numpy as np
import pytest

from paper_2608_02691_amd import int2kv as K

GIB = 1 << 30


@pytest.mark.parametrize("hq,h", [(32, 8), (40, 8), (8, 8), (64, 1), (128, 128)])
def test_whole_prompts_are_bounded(hq, h):
    for n in (32768, 131072, 262144, 1 << 20):
        # a chunk of 32 row tiles: 17 KiB operands a tile, 8 bytes a row and range, sums of a chunk and running ones
        ranges = n // 256
        least = h * 32 * 17 * 1024 + ranges * 32 * h * 32 * 8 + 2 * h * n * 4
        assert K.int2kv_token_weights_workspace_bytes(1, hq, h, n, n, n) <= max(GIB, least + 4096), n


def test_batches_of_prompts_are_bounded_by_a_chunk_each():
    for B in (4, 16, 64):
        n, h = 65536, 8
        least = B * h * (32 * 17 * 1024 + (n // 256) * 32 * 32 * 8 + 2 * n * 4)
        assert K.int2kv_token_weights_workspace_bytes(B, 32, h, B * n, n, n) <= max(GIB, least + 4096)


def test_calls_below_the_bound_keep_their_sizes():
    """Prompts whose operands and statistics have room at once: 17 KiB a row tile of a KV head, 8 bytes a row and range."""
    for B, n in ((1, 4096), (4, 4096), (1, 16384)):
        tiles = B * n * 4 // 32 + B + 1
        need = K.int2kv_token_weights_workspace_bytes(B, 32, 8, B * n, n, n)
        assert need >= tiles * 8 * (17 * 1024 + (n // 256) * 32 * 8) and need < GIB


def test_workspaces_around_the_bound_serve_every_smaller_call():
    rng = np.random.default_rng(5)
    top = 0
    for hq, h in ((32, 8), (40, 8), (8, 8), (64, 1), (64, 64)):
        for _ in range(400):
            big = [int(x) for x in np.exp(rng.uniform([0, 7, 5, 7], [4, 13, 12.5, 13.5]))]  # batch, total_q, max_q, max_ctx
            small = [max(int(i == 0), int(x * rng.uniform(0, 1) ** rng.choice([0.1, 0.5]))) for i, x in enumerate(big)]
            need = K.int2kv_token_weights_workspace_bytes(big[0], hq, h, *big[1:])
            top += need >= GIB
            assert need >= K.int2kv_token_weights_workspace_bytes(small[0], hq, h, *small[1:]), (hq, h, big, small)
    assert top > 100
