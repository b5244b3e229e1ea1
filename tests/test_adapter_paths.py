"""The ways that calls of adapters go at the sizes of the GPU tests, on the CPU: what these tests are
for is what they run."""
import test_gpu_adapter_few as few
import test_gpu_adapter_loops as loops
import test_gpu_adapter_order as order
from adapter_grids import adapter_grids

CHUNK = 2048                          # tokens of factors_kernel's chunk


def _most_tiles(T, L, tile, columns):
    some = min(T, L)
    return ((some + (T - some) // tile) * columns + 7) // 8 * 8


def test_both_ways_are_run():
    sizes = [(T, order.L, r, order.N, order.D) for T, r in order.BOTH]
    got = dict(zip(sizes, adapter_grids([(0, *s) for s in sizes])))
    kernels = set()
    for (T, *rest), launched in got.items():
        names = [name for name, _ in launched]
        if T == order.FEW:
            assert all(name.startswith("few_") for name in names), (T, rest, names)
        else:
            assert names[0] == "order_kernel<false>", (T, rest, names)
            kernels |= set(names)
    for want in ("shrink_kernel<1, 1>", "shrink_kernel<1, 2>", "shrink_tile_kernel<4, 32>",
                 "shrink_tile_kernel<8, 32>", "expand_kernel<2, 1>", "expand_kernel<2, 2>",
                 "expand_tile_kernel<4>", "expand_tile_kernel<8>"):
        assert want in kernels, want
    tuned = adapter_grids([(0, T, 4, 24, 272, 400) for T in order.TUNED])
    assert [one[0][0].startswith("order_") for one in tuned] == [True, False, False]


def test_many_columns_are_more_than_a_waves_first():
    cases = [(0, *s) for s in loops.WIDE] + [(1, *s) for s in loops.WIDE_BACK]
    seen = set()
    for (backward, T, L, r, n, d), launched in zip(cases, adapter_grids(cases)):
        (name, (groups, *_)), = [g for g in launched if g[0].startswith("expand_kernel")]
        rest = -(-T // 64)
        # fewer workgroups than with 128 columns each, of which a wave has 32
        assert groups - rest < _most_tiles(T, L, 32, -(-(d if backward else n) // 128)), (T, L, r, n, d)
        seen.add((backward, name))
    assert seen == {(b, f"expand_kernel<2, {j}>") for b in (0, 1) for j in (1, 2)}


def test_an_adapter_has_more_tokens_than_a_chunk():
    seen = set()
    for s, launched in zip(loops.HEAVY, adapter_grids([(1, *s) for s in loops.HEAVY])):
        (name, (_, splits, _)), = [g for g in launched if g[0].startswith("factors_kernel")]
        T, L, r, *_ = s
        ids = loops.heavy_ids(T, L, r)
        assert splits == 1 and int((ids == 5).sum()) > CHUNK and not (ids == 9).any(), s
        seen.add(name)
    assert seen == {f"factors_kernel<{j}>" for j in (1, 2, 4, 8)}


def test_few_tokens_in_one_launch_or_two():
    got = adapter_grids([(0, *s) for s in few.ONE + few.TWO])
    names = [[name for name, _ in launched] for launched in got]
    for s, launched in zip(few.ONE + few.TWO, names):
        assert launched == (["few_kernel"] if s in few.ONE else ["few_shrink_kernel", "few_expand_kernel"]), s
