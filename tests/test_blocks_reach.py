"""The shapes of the tests that are about a kernel of the linear layers by blocks, and not about a size, reach all of these kernels."""
import pytest

from test_blocks_plan import kernel_of, plan  # noqa: F401  (a fixture)

KERNELS = [("pair",), ("wide",), ("middle",)] + [("narrow", ks) for ks in (1, 2, 4)] + [("few", h, ks) for h in (16, 32, 64) for ks in (1, 2)] + [("few", 64, 4), ("few", 16, 4), ("few", 16, 8)]


def taken(plan, scaled, grouped):
    return ({("scaled",) + kernel_of(plan(m, n, -(-k // 128))) for m, n, k in scaled} |
            {("grouped",) + kernel_of(plan(sum(c), n, -(-k // 64), len(c), False)) for c, n, k in grouped} |
            {("grouped_scaled",) + kernel_of(plan(sum(c), n, -(-k // 128), len(c), True)) for c, n, k in grouped})


@pytest.mark.parametrize("op", ["scaled", "grouped", "grouped_scaled"])
def test_waits_that_run_out(plan, op):  # noqa: F811
    import test_gpu_blocks_waits as T
    seen = taken(plan, T.SCALED, T.GROUPED)
    assert not [k for k in KERNELS if (op,) + k not in seen]


@pytest.mark.parametrize("op", ["grouped", "grouped_scaled"])
def test_rows_of_nobody(plan, op):  # noqa: F811
    """The same shapes with the rows in front of the first expert and behind the last."""
    import test_gpu_blocks_every_kernel as T
    seen = set()
    for c, n, k in T.GROUPED:
        f8 = op == "grouped_scaled"
        seen.add((op,) + kernel_of(plan(sum(c) + T.LEAD + T.REST, n, -(-k // (128 if f8 else 64)), len(c), f8)))
    assert not [k for k in KERNELS if (op,) + k not in seen]


def test_long_sums(plan):  # noqa: F811
    """Every width of bf16, and operands exchanged at every height."""
    import test_gpu_blocks_every_kernel as T
    seen = {kernel_of(plan(sum(c), n, -(-k // 64), len(c), False))[:2] for c, n, k in T.LONG}
    assert {("few", 16), ("few", 32), ("few", 64), ("pair",), ("wide",), ("middle",)} <= seen and any(k[0] == "narrow" for k in seen)
