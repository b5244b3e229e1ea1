"""The forms that calls on groups of rows and adapters of given sizes run: those that the GPU tests name
are the ones that they get, and every form is one that a GPU test runs."""
import test_gpu_adapters
import test_gpu_grouped
from group_launches import group_launches

LINEAR = {"64x32 x 2": "tile_kernel<0, 64, 32, 4, 1, 3, 64, 2>",
          "64x32": "tile_kernel<0, 64, 32, 4, 1, 4, 64, 1>", "64x64": "tile_kernel<0, 64, 64, 2, 2, 3, 64, 1>",
          "128x64": "tile_kernel<0, 128, 64, 2, 2, 3, 64, 1>", "turns": "turns_kernel<0>"}
GRAD_X = {"64x32 x 2": "tile_kernel<1, 64, 32, 4, 1, 3, 64, 2>",
          "64x32": "tile_kernel<1, 64, 32, 4, 1, 4, 64, 1>", "64x64": "tile_kernel<1, 64, 64, 2, 2, 3, 64, 1>",
          "128x64": "tile_kernel<1, 128, 64, 2, 2, 3, 64, 1>",
          "turns": "turns_kernel<1>"}
GRAD_W = {"128x64": "tile_kernel<2, 128, 64, 2, 2, 3, 32, 1>",
          "128x128": "tile_kernel<2, 128, 128, 2, 2, 3, 32, 1>",
          "256x256": "tile_kernel<2, 256, 256, 2, 4, 4, 32, 1>", "turns": "turns_kernel<2>"}
OF = {"linear": LINEAR, "x": GRAD_X, "w": GRAD_W}


def test_product_forms_are_as_named():
    cases = test_gpu_grouped.FORMS
    got = group_launches([(what, sum(c), len(c), n, k) for what, _, c, n, k in cases])
    seen = set()
    for (what, form, c, n, k), names in zip(cases, got):
        assert names[0] == OF[what][form], (what, form, c, n, k, names)
        assert names[1:] == ([f"join_kernel<{'linear x w'.split().index(what)}>"]
                             if form == "turns" else [])
        seen.add(names[0])
    assert seen == {name for forms in OF.values() for name in forms.values()}


def test_many_tiles_are_not_split():
    for what, name in (("linear", "turns_kernel<0>"), ("x", "turns_kernel<1>")):
        (names,) = group_launches([(what, 1 << 19, 8, 4096, 4096)])
        assert names == [name]


def test_order_in_one_launch_or_two():
    got = group_launches([("order", 1, 1, 1), ("order", 512, 8, 256), ("order", 4097, 1, 63)])
    assert got == [["order_kernel<false>"], ["order_kernel<false>"],
                   ["order_count_kernel", "order_kernel<true>"]]


def test_adapter_forms():
    cases = [("adapters", *s) for s in test_gpu_adapters.SHAPES] + \
        [("backward", *s) for s in test_gpu_adapters.SHAPES]
    got = group_launches(cases)
    kernels = {n for names in got for n in names}
    # few tokens: in one launch and in two; many: every width of the rank's tiles
    for want in ("few_kernel", "few_shrink_kernel", "few_expand_kernel", "transpose_kernel",
                 "sum_parts_kernel", *(f"factors_kernel<{j}>" for j in (1, 2, 4, 8)),
                 "shrink_kernel<1, 1>", "shrink_kernel<1, 2>", "shrink_tile_kernel<4, 32>",
                 "shrink_tile_kernel<8, 32>", "shrink_tile_kernel<4, 64>", "shrink_tile_kernel<8, 64>",
                 "expand_kernel<2, 1>", "expand_kernel<2, 2>", "expand_tile_kernel<4>",
                 "expand_tile_kernel<8>"):
        assert want in kernels, want
    few = []
    for (what, T, *rest), names in zip(cases, got):
        if what == "adapters" and names[0].startswith("few_"):
            assert names in (["few_kernel"], ["few_shrink_kernel", "few_expand_kernel"]) and T <= 256
            few.append((T, *rest))
        elif what == "adapters":
            assert names[-3 if T <= 4096 else -4].startswith("order_") and len(names) in (3, 4)
    assert (1, 3, 8, 8, 8) in few and (256, 8, 24, 264, 520) in few
    assert (257, 8, 24, 264, 520) not in few and (200, 3, 128, 1032, 72) not in few


def test_columns_of_one_buffer_do_not_overlap():
    cases = [("beside", 8, 40, 64, 104, 64), ("beside", 8, 40, 64, 104, -40),
             ("beside", 8, 40, 64, 128, 88), ("beside", 8, 40, 64, 104, 4 * 104 + 64),
             ("beside", 8, 40, 64, 104, 7 * 104 + 64), ("beside", 8, 40, 64, 64, 8 * 64),
             ("beside", 8, 64, 64, 64, -8 * 64)]
    assert all(len(names) == 1 for names in group_launches(cases))
