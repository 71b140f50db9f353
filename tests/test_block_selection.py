"""Which kernel a product of 8-bit matrices takes: that the cases of test_gpu_block_tiles.py run what they say, and what the rules are to keep."""
import pytest

from paper_1705_05249_amd import experts as X
from tests import test_gpu_block_tiles as T
from tests.block_choice import choices


def problem(case):
    mode, kernel, sums, m, n, k, _ = case
    lead, start = T.leading(case)
    experts = {"dense": 0, "rows": T.FIVE, "sum": T.TWO}[mode]
    need = {"dense": lambda: X.mg_block_gemm_workspace_bytes(m, n, k), "rows": lambda: X.mg_block_gemm_grouped_workspace_bytes(experts, m, n, k),
            "sum": lambda: X.mg_block_gemm_grouped_sum_workspace_bytes(experts, k, m, n)}[mode]()
    return dict(mode=mode, m=m, n=n, k=k, pow2=sums.endswith("pow2"), fp32=sums in T.FP32_SUMS, b_square=sums == "square", groups=experts, lda=lead, ldb=lead, start=start,
                workspace=need)


def test_the_cases_run_the_kernels_they_name():
    cases = T.DENSE + T.ROWS + T.SUM
    for case, (kernel, sums, slices, _) in zip(cases, choices([problem(c) for c in cases])):
        assert (kernel, sums, slices > 1) == (case[1], case[2], case[6]), (case, kernel, sums, slices)


def test_every_kernel_has_a_case():
    """aligned tiles and those for any address, every way of summing that a call of the mode can ask for"""
    every = ("pow2", "any", "square", "fp32", "fp32 pow2")
    for cases, sums in ((T.DENSE, every), (T.ROWS, every), (T.SUM, ("pow2", "any", "fp32", "fp32 pow2"))):
        for kernel in ("256", "128", "any 128"):
            assert {c[2] for c in cases if c[1] == kernel} == set(sums), (cases[0][0], kernel)
    assert {c[2] for c in T.ROWS if c[1] == "few"} == set(every)


def test_indexed_rows_are_as_far_apart_as_tokens():
    """rows fetched by slot / fan: A has a row for each token, and only its size decides whether 32-bit offsets reach them"""
    many = dict(mode="rows", m=65536 * 8, n=2048, k=4096, groups=64, fan=8, pow2=True, b_square=True, indexed=True)
    assert choices([many])[0][0] == "256"                                       # A spans 2^28 bytes
    last = (1 << 31) - (1 << 20) - 4096                                         # from there on offsets do not fit
    rows = {fan: fan * (last // 4096) for fan in (1, 3, 64)}
    for fan, m in rows.items():
        fits, beyond = choices([dict(many, m=m - fan, fan=fan), dict(many, m=m + fan + 1, fan=fan)])
        assert fits[0] == "256" and beyond[0].startswith("any"), fan


@pytest.mark.parametrize("groups,n,mean,kernel", (
    (4, 2048, 1, "few"), (4, 2048, 12, "few"), (8, 2048, 8, "few"), (8, 2048, 12, "64"), (16, 2048, 2, "64"), (32, 2048, 1, "64"), (64, 2048, 16, "64"), (128, 1024, 1, "64"),
    (256, 512, 4, "64"), (16, 1000, 8, "few"), (4, 7168, 2, "64"), (64, 200, 2, "few"), (32, 2048, 17, "64")))
def test_few_rows_of_experts(groups, n, mean, kernel):
    """tiles where all experts together have enough of them for the chip: they read an expert's weights once, however many of the rows it has"""
    for lda in (4096, 4099):
        got = choices([dict(mode="rows", m=mean * groups, n=n, k=4096, groups=groups, pow2=True, b_square=True, lda=lda, ldb=lda)])[0][0]
        assert got == (kernel if lda == 4096 or kernel == "few" else "any 64"), got
