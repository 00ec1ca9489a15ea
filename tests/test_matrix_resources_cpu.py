"""What the compiler made of the kernels for tokens' scores and orthogonalised matrices: those whose
speed rests on registers use no scratch memory, and no more registers than their share of a CU."""
import pytest

from test_kernel_resources_cpu import kernels, named  # noqa: F401 (kernels is a fixture)


def test_scratch(kernels):  # noqa: F811
    seen = 0
    for name, k in kernels.items():
        if "score_" not in name and "matrix_" not in name:
            continue
        seen += 1
        assert k[".private_segment_fixed_size"] == 0, (name, k[".private_segment_fixed_size"])
    assert seen > 80


# (part of the name, wavefronts a SIMD that the kernel's registers have to leave room for)
@pytest.mark.parametrize("part,waves", [("score_rowsILi1ELi512ELi8E", 8), ("score_rowsILi1ELi512ELi13E", 5), ("score_rowsILi0ELi1024ELi13E", 4),
                                        ("score_gradientILi1ELi1024E", 8), ("matrix_productILi2ELi4E", 2), ("matrix_productILi1ELi3E", 3),
                                        ("matrix_smallI", 4)])
def test_registers(kernels, part, waves):  # noqa: F811
    for k in named(kernels, part):
        assert (k[".vgpr_count"] + 7) // 8 * 8 <= 512 // waves, (k[".name"], k[".vgpr_count"])
