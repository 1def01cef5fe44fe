"""Which kernel a product with a head in 8-bit integers takes: the sizes of the GPU tests reach every one of them."""
from paper_2505_24034_amd import binding
from test_gpu_row_head import PRODUCTS

DIRECT, DEEP, T64, T128, T256 = range(5)


def test_every_kernel_is_among_the_tested_products():
    rules = binding._load_native()
    assert {rules.row_plan(N, V, d)[0] for N, V, d in PRODUCTS} == {DIRECT, DEEP, T64, T128, T256}
    plans = [(V, rules.row_logits_plan(N, V, d)) for N, V, d in PRODUCTS]
    assert {p[0] for _, p in plans} == {DIRECT, DEEP, T64, T128, T256}
    assert any(p[1] < V and p[2] != p[0] for V, p in plans)                # rows behind the whole rounds in a launch of their own


def test_rows_of_the_first_launch():
    rules = binding._load_native()
    for N in (65, 129, 300, 900, 1900, 4096):
        for V in (1000, 8191, 33001, 65066, 128256):
            for d in (16, 528, 2048, 8192):
                tile, rows, rest = rules.row_logits_plan(N, V, d)
                assert 0 < rows <= V and (rows == V or rows % 256 == 0 and tile == T256 and rest != T256)
