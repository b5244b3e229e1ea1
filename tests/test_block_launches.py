"""The forms of block_linear and block_experts that calls of given sizes run: every form is one that a
GPU test runs, and the forms that those tests name are the ones they get."""
import pytest

import test_gpu_block_error
import test_gpu_block_forms
import test_gpu_blocks
from block_launches import block_launches

LINEAR = {"16x16": "product_kernel<0, 1, 1, 4>", "32x16": "product_kernel<0, 2, 1, 4>",
          "16x32": "product_kernel<0, 1, 2, 4>", "32x32": "product_kernel<0, 2, 2, 4>",
          "64x32": "tile_kernel<0, 64, 32, 2, 2, 4, false>",
          "64x64": "tile_kernel<0, 64, 64, 2, 2, 3, false>",
          "128x64": "tile_kernel<0, 128, 64, 4, 2, 5, false>",
          "128x128": "tile_kernel<0, 128, 128, 2, 4, 4, false>",
          "128x256": "tile_kernel<0, 128, 256, 2, 4, 3, false>",
          "256x256": "tile_kernel<0, 256, 256, 2, 4, 2, false>"}
QUANTISE, COMBINE = "quantize_rows_kernel<", "combine_kernel"
# gate/up and down of the experts by the names that the tests give them
UP = {"few": "product_kernel<1, 2, 1, 4>", "32": "tile_kernel<1, 256, 32, 8, 1, 4, true>",
      "128": "tile_kernel<1, 256, 128, 4, 2, 3, true>",
      "128 in FP8": "tile_kernel<1, 256, 128, 4, 2, 3, false>"}
DOWN = {"few": "product_kernel<2, 2, 1, 4>", "32": "tile_kernel<2, 256, 32, 8, 1, 4, false>",
        "64": "tile_kernel<2, 128, 64, 4, 2, 5, false>",
        "128": "tile_kernel<2, 256, 128, 4, 2, 3, false>"}
ONE = ["small_kernel<1, 2, 8, 1>", "small_kernel<2, 1, 8, 1>"]
# test_linear_forms' label of this case is another form's than the rule's choice
NOT_AS_NAMED = {("16x32", 30, 2049, 400): "32x16"}


def _cases(test):
    """The parameters of a parametrised test."""
    (mark,) = [m for m in test.pytestmark if m.name == "parametrize"]
    return [tuple(c) for c in mark.args[1]]


def test_linear_forms_are_as_named():
    cases = _cases(test_gpu_blocks.test_linear_forms) + _cases(test_gpu_block_forms.test_linear)
    got = block_launches([("linear", T, n, k, True) for _, T, n, k in cases])
    for case, names in zip(cases, got):
        assert names == [LINEAR[NOT_AS_NAMED.get(case, case[0])]], case
    # and every form is run
    assert {names[0] for names in got} == set(LINEAR.values())


def test_linear_quantises_its_rows_itself_or_first():
    sizes = [(1, 4095, 16384), (16, 4096, 1024), (17, 300, 656), (16, 300, 1040)]
    got = block_launches([("linear", T, n, k, False) for T, n, k in sizes])
    assert got[0] == ["small_kernel<0, 1, 4, 1>"] and got[1] == ["small_kernel<0, 1, 4, 2>"]
    for names in got[2:]:
        assert len(names) == 2 and names[0].startswith(QUANTISE) and names[1] in LINEAR.values()


@pytest.mark.parametrize("test", [test_gpu_blocks.test_experts_forms,
                                  test_gpu_block_error.test_error_of_the_whole_output],
                         ids=["forms", "error"])
def test_experts_forms_are_as_named(test):
    cases = _cases(test)
    got = block_launches([("experts", *c[1:]) for c in cases])
    for (forms, *sizes), names in zip(cases, got):
        if forms == "one token":
            assert names == ONE, sizes
            continue
        up, down = forms.split(" / ")
        # (the first of the two tests does not name the instructions)
        ups = {UP[up], UP["128 in FP8"]} if test.__name__ == "test_experts_forms" and up == "128" \
            else {UP[up]}
        assert names[1] in ups, (forms, sizes, names)
        assert names[0] == "prepare_kernel" and names[-2:] == [DOWN[down], COMBINE], (forms, names)
        assert len(names) == (5 if up == "few" else 4)
        assert (up == "few") == names[2].startswith(QUANTISE)


def test_every_experts_form_is_run():
    cases = (_cases(test_gpu_blocks.test_experts_forms)
             + _cases(test_gpu_block_error.test_error_of_the_whole_output))
    seen = {n for names in block_launches([("experts", *c[1:]) for c in cases]) for n in names}
    assert set(UP.values()) | set(DOWN.values()) | set(ONE) <= seen
