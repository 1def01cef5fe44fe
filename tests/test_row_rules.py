"""Which kernel a product with a head in 8-bit integers takes: the sizes of the GPU tests reach every one of them."""
import pytest

from paper_2505_24034_amd import binding
from test_gpu_row_head import PRODUCTS

DIRECT, T64, T128, T256 = range(4)


@pytest.mark.parametrize("logprobs", [0, 1])
def test_every_kernel_is_among_the_tested_products(logprobs):
    rules = binding._load_native()
    plans = [(V, *rules.row_plan(N, V, d, logprobs)[:3]) for N, V, d in PRODUCTS]
    assert {p[1] for p in plans} == {DIRECT, T64, T128, T256}
    rests = {p[3] for p in plans if p[2] < p[0]}                           # rows behind the whole rounds, in a launch of their own
    assert rests >= {T64, T128}


def test_rows_of_the_first_launch_and_room_for_the_partials():
    rules = binding._load_native()
    for N in (1, 4, 16, 17, 64, 65, 129, 300, 900, 1900, 4096, 16384):
        for V in (1, 63, 1000, 8191, 16032, 33001, 65066, 128256, (1 << 21) - 1):
            for d in (16, 528, 2048, 8192, 131056):
                for logprobs in (0, 1):
                    tile, rows, rest, partials, floats = rules.row_plan(N, V, d, logprobs)
                    assert 0 < rows <= V and (rows == V or rows % 256 == 0 and tile == T256 and rest in (T64, T128, T256)), (N, V, d)
                    assert N <= 16 or DIRECT not in (tile, rest)
                    assert partials * (-(-N // 64) * 64) <= floats, (N, V, d)
