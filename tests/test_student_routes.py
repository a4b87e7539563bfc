"""Which kernels the student nets' operators take, and with what grids."""
import pytest

from tests import student_routes as R


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    with pytest.MonkeyPatch.context() as m:
        yield R.build(tmp_path_factory.mktemp("routes"), m)


def test_grids_have_fewer_than_2_to_the_32_threads(program):
    """Sizes that a card's memory holds, of the most rows, the most columns, and every kernel's border between."""
    most_rows, elements = 1 << 28, 1 << 36
    cases = []
    for cols in (1, 7, 512, 513, 1024, 1025, 4096, 4097, 8192, 8193, 16384, 16385, 1 << 20):
        rows = min(most_rows, elements // cols)
        for type_ in ("f32", "bf16"):
            cases += [("norm", rows, cols, type_, out) for out in ("-", "e4m3", "e4m3_128")]
            cases += [("norm_back", rows, cols, type_, kept, wanted) for kept in ("-", "e4m3") for wanted in ("dx", "all")]
            cases += [("distil", rows, cols, min(cols, 9), type_, wanted) for wanted in ("loss", "all")]
            cases += [("load", rows, cols, type_, kind) for kind in ("rows", "tiles")]
            rows_along = min(rows, 1 << 23)              # (a product's rows are a transposed matrix's columns)
            cases += [("save", rows_along, cols, type_, kind, which) for kind in ("rows", "tiles") for which in ("out", "out_t", "both")]
            cases += [("product", rows_along, cols, inputs, type_, x, y) for inputs in (1, 129, 8192) for x in ("-", "e4m3_128") for y in ("-", "e4m3_128")]
            cases += [("product_back", rows_along, cols, inputs, type_, wanted) for inputs in (1, 129, 8192) for wanted in ("dx", "dw", "all")]
    wrong = [(case, k) for case, launches in zip(cases, R.kernels(program, cases)) for k in launches if k[2] * k[3] >= 1 << 32]
    assert not wrong, "\n".join(map(str, wrong))


def test_backward_passes_of_products_go_the_ways_they_name(program):
    for type_ in ("bf16", "f32"):
        cases = [("product_back", *sizes, type_, "all") for sizes, _ in R.BACKWARD]
        got = [(sizes, R.describe_backward(sizes, k)) for (sizes, _), k in zip(R.BACKWARD, R.kernels(program, cases))]
        assert got == R.BACKWARD


def test_layer_norms_take_the_kernels_they_name(program):
    for type_ in ("bf16", "f32"):
        for kept in ("-", "e4m3"):
            for want, sizes in R.NORM_BACK.items():
                for launches in R.kernels(program, [("norm_back", *s, type_, kept, "all") for s in sizes]):
                    named = [f"{kernel}, {threads if kernel != 'k_layer_backward' else args[2]} threads" for kernel, args, _, threads in launches]
                    assert want in named, (want, sizes, named)
                    assert ("k_layer_finish, 1024 threads" in named) == ("few" not in want)
