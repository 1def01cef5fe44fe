"""Which kernel logits of one or two tokens take where 64 x 64 tiles of W leave half of the chip without work, walked on the CPU."""
import pytest

from paper_2505_24034_amd import binding as L

DIRECT, TILES_64 = 0, 2


@pytest.mark.parametrize("N,V,d,kernel", [(1, 32641, 4096, DIRECT), (1, 34500, 2048, DIRECT), (2, 34500, 8192, DIRECT), (1, 40960, 1024, DIRECT),
                                          (2, 36000, 4096, DIRECT), (1, 40961, 4096, TILES_64), (3, 34500, 4096, TILES_64), (1, 34500, 512, TILES_64),
                                          (1, 34500, 1536, TILES_64), (1, 34500, 6144, TILES_64), (2, 50000, 4096, TILES_64), (1, 128256, 4096, TILES_64)])
def test_one_or_two_tokens(N, V, d, kernel):
    rules = L._load_native()
    assert rules.block_logits_plan(N, V, d) == (kernel, V, kernel)
    assert rules.block_plan(N, V, d, 0)[0] == TILES_64                     # log-probabilities stay on tiles


def test_what_was_direct_stays_so():
    rules = L._load_native()
    for N in (1, 2, 4):
        for V in (1, 1000, 16032, 32640):
            for d in (16, 512, 1536, 4096):
                assert rules.block_logits_plan(N, V, d)[0] == rules.block_plan(N, V, d, 0)[0] == DIRECT


def test_no_workspace_for_sizes_that_no_call_takes():
    size = L.logprobs_blocks_workspace_bytes
    for N, V in ((1, 1 << 21), (1 << 27, 5), (1 << 62, 1 << 62), (-1, 5), (5, -1)):
        assert size(N, V) == 0, (N, V)
    assert size((1 << 27) - 1, 5) >= size(1 << 20, 5) > 0 and size(5, (1 << 21) - 1) >= size(5, 1 << 20) > 0
