"""The rules that pick a kernel for a product with an 8-bit head, walked on the CPU: whatever they pick, its partials fit the workspace, and
a workspace of a larger call serves a smaller one."""
import pytest

from paper_2505_24034_amd import binding as L

TOKENS = sorted({1, 2, 4, 5, 16, 17, 63, 64, 65, 127, 128, 129, 300, 348, 1041, 2299, 9937, 16384} | {64 * k + o for k in range(1, 40, 3) for o in (-1, 0, 1)})
VOCAB = sorted({1, 15, 16, 17, 64, 65, 127, 129, 1000, 1766, 4346, 8000, 8191, 8192, 8193, 16032, 32640, 32641, 33001, 65408, 65409, 128256} |
               {128 * k + o for k in range(1, 60, 5) for o in (-1, 0, 1)})


@pytest.fixture(scope="module")
def rules():
    return L._load_native()


def test_partials_fit_whatever_is_picked(rules):
    seen = set()
    for N in TOKENS:
        for V in VOCAB:
            for d in (16, 512, 528, 1024, 2064, 4096):
                kernel, rows, plane = rules.block_plan(N, V, d, 0)
                seen.add(kernel)
                assert -(-V // rows) * (-(-N // 64) * 64) <= plane, (N, V, d)
                assert kernel > 1 or N <= (16 if kernel == 0 else 64)      # the two for few tokens hold no more
                assert rules.block_plan(N, V, d, 1)[0] <= 3                # fp32 logits: tiles of 128 rows at most
    assert seen == {0, 1, 2, 3, 4}


def test_planes_do_not_shrink(rules):
    size = {(n, v): rules.block_plan(n, v, 512, 0)[2] for n in TOKENS for v in VOCAB}
    for v in VOCAB:
        assert all(size[a, v] <= size[b, v] for a, b in zip(TOKENS, TOKENS[1:]))
    for n in TOKENS:
        assert all(size[n, a] <= size[n, b] for a, b in zip(VOCAB, VOCAB[1:]))


def test_logits_cover_every_row_once(rules):
    split = 0
    for N in TOKENS:
        for V in VOCAB:
            for d in (16, 528, 2048, 8192):
                first, rows, rest = rules.block_logits_plan(N, V, d)
                assert rows == V or (0 < rows < V and rows % 256 == 0 and first == 4 and rest in (2, 3)), (N, V, d)
                assert first > 1 or N <= (16 if first == 0 else 64)
                split += rows < V
    assert split > 0
