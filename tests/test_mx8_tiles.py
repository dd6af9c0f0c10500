"""CPU-only: the sizes at which the GPU tests compare the 8-bit experts with the oracle reach the kernels they are there for."""
import ctypes

from paper_2112_14397_amd import binding as B
import test_gpu_mx8_experts as mx8


def tiles(shape, announced_pairs, num_cu=256):
    """Rows x columns / waves of both products; the library answers on the host, by the rule its launchers use."""
    out = []
    for name in ("ffn_mx8_gemm1", "ffn_mx8_gemm2"):
        t = (ctypes.c_int * 3)()
        assert B.lib().evomoe_test_ffn_tile(ctypes.byref(shape), num_cu, ctypes.c_int64(announced_pairs),
                                            B.KERNEL_IDS.index(name), t) == 1
        out.append("%dx%d/%d" % tuple(t))
    return tuple(out)


def test_cases_reach_the_tiles_they_name_and_all_there_are():
    seen = [set(), set()]
    for T, d, E, F, P, *named in mx8.CASES + mx8.LARGE:
        got = tiles(B.make_shape(T, d, E, F, "bf16", "gelu", P + 37), P)
        assert got == tuple(named), (T, d, E, F, P)
        for s, t in zip(seen, got):
            s.add(t)
    assert seen == [{"32x32/4", "64x128/4", "128x128/4", "256x256/8"}, {"32x32/4", "64x64/4", "64x128/4", "128x128/4", "192x128/4", "256x256/4"}]
