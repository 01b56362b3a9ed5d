"""The shapes that the fused products are tested at take the kernels that they are named for."""
from gemm_kernels import kernel_of
from linear_cases import FRAGMENTS, GLU_SHAPES
from test_launch_plans import gemm, plans  # noqa: F401


def test_every_kernel_is_reached(plans):  # noqa: F811
    for shapes in (FRAGMENTS, GLU_SHAPES):
        for name, (M, N, K) in shapes.items():
            bits = int(name[0])
            assert kernel_of(gemm(plans, M, N, K, bits, True), M, bits, True) == name, (name, M, N, K)
