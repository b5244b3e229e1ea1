"""The ways that calls of adapters go at the sizes of the GPU tests, on the CPU: what these tests are
for is what they run."""
import test_gpu_adapter_order as order
from adapter_grids import adapter_grids

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
