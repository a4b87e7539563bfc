"""The kernels that the GPU tests of the products mean to run are the ones that run, and none is left out."""
import pytest

from tests import operator_routes as R


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    with pytest.MonkeyPatch.context() as m:
        yield R.build(tmp_path_factory.mktemp("routes"), m)


def test_cases_take_the_kernels_they_name(program):
    wrong = [(case, want, got) for (case, want), launches in zip(R.CASES, R.kernels(program, [c for c, _ in R.CASES]))
             if (got := R.describe(case, launches)) != want]
    assert not wrong, "\n".join(map(str, wrong))


def test_cases_take_every_kernel(program):
    mine = ("k_product", "k_both", "k_few", "k_slope", "k_join", "k_join_all", "k_column_finish")
    have = {(name, tuple(args)) for name, args in R.of_library(program) if name in mine}
    run = {(name, tuple(args)) for launches in R.kernels(program, [c for c, _ in R.CASES]) for name, args, _, _ in launches}
    assert len(have) > 80 and run == have, f"{sorted(have - run)}"


def test_single_rows_forward(program):
    """A few rows take the kernel that streams the weights, whatever the other sizes."""
    cases = [("forward", rows, o, i, t, "-") for rows in (1, 4) for o in (1, 9, 5000) for i in (1, 9, 5000) for t in ("f32", "bf16")]
    assert all(R.describe(c, k)[0].endswith("waves") and len(k) == 1 for c, k in zip(cases, R.kernels(program, cases)))
