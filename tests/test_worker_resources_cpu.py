"""What the compiler made of the worker-side operators' kernels: those whose speed
rests on holding their values in registers keep them there (no scratch memory)."""
import pytest

from test_kernel_resources_cpu import kernels, named  # noqa: F401 (kernels is a fixture)


@pytest.mark.parametrize("part", [
    "dropout_kernelILi1ELb1ELi4E", "dropout_kernelILi1ELb0ELi1E",
    # element type 1 (bfloat16) and 0; vectors a thread; groups in a vector
    "norm_forward_foldILi1ELi4ELi1E", "norm_forward_foldILi1ELi8ELi1E", "norm_forward_foldILi1ELi16ELi1E",
    "norm_forward_foldILi1ELi8ELi4E", "norm_forward_foldILi0ELi16ELi1E", "norm_backward_foldILi1ELi2ELi1E",
    "norm_backward_foldILi1ELi4ELi1E", "norm_backward_foldILi1ELi8ELi1E", "norm_backward_foldILi1ELi8ELi2E",
    "norm_back_sumsILi1E", "norm_backward_splitILi1E", "norm_momentsILi1E", "norm_forward_splitILi1E",
    # threads a row; vectors a thread
    "policy_heldILi1ELi64ELi8E", "policy_heldILi1ELi512ELi13E", "policy_heldILi2ELi512ELi13E",
    "policy_heldILi0ELi512ELi13E", "pref_logpILi1ELi256E", "pref_gradientILi1ELi1024ELb0E",
])
def test_no_scratch(kernels, part):  # noqa: F811
    for k in named(kernels, part):
        assert k[".private_segment_fixed_size"] == 0, (k[".name"], k[".private_segment_fixed_size"])


def test_held_rows_leave_room_for_two_workgroups_on_a_cu(kernels):  # noqa: F811
    # 512 threads are 2 wavefronts on each of a CU's 4 SIMDs, which have 512 registers a lane
    for k in named(kernels, "policy_heldILi1ELi512ELi13E"):
        assert k[".vgpr_count"] <= 128, k[".vgpr_count"]
