"""Scratch memory of every kernel of the worker-side operators: none, or a few registers'
worth where the values a thread holds leave too few of its 128 registers, and no more
than that."""
import pytest

from test_kernel_resources_cpu import kernels  # noqa: F401 (a fixture)

# bytes a thread, by part of the name: element type (1 bfloat16, 2 float16), threads a row or vectors
# a thread, then vectors a thread or groups in a vector
SPILLS = {
    "policy_heldILi1ELi512ELi26E": 68, "policy_heldILi2ELi512ELi26E": 68,      # 16-bit rows of 6,657 to 13,312 vectors
    "policy_heldILi0ELi1024ELi20E": 20, "policy_heldILi1ELi1024ELi20E": 20, "policy_heldILi2ELi1024ELi20E": 20,
    "norm_forward_foldILi1ELi16ELi8E": 48, "norm_forward_foldILi2ELi16ELi8E": 48,  # one channel a group
    "norm_backward_foldILi1ELi8ELi4E": 24, "norm_backward_foldILi2ELi8ELi4E": 24,  # two
    "norm_backward_foldILi1ELi8ELi8E": 88, "norm_backward_foldILi2ELi8ELi8E": 88,  # one
    "norm_forward_heldILi1ELi8ELi16E": 44, "norm_forward_heldILi2ELi8ELi16E": 44,  # groups of other widths
    "norm_backward_heldILi1ELi8ELi8E": 108, "norm_backward_heldILi2ELi8ELi8E": 108,
}
OURS = ("dropout_kernel", "norm_forward_", "norm_backward_", "norm_moments", "norm_join", "norm_back_", "norm_params", "policy_", "pref_")


def test_scratch_of_every_kernel(kernels):  # noqa: F811
    seen = {part: 0 for part in SPILLS}
    for name, k in kernels.items():
        if not any(part in name for part in OURS):
            continue
        most = 0
        for part, bytes_ in SPILLS.items():
            if part in name:
                most, seen[part] = bytes_, seen[part] + 1
        assert k[".private_segment_fixed_size"] <= most, (name, k[".private_segment_fixed_size"])
    assert all(n == 1 for n in seen.values()), seen


@pytest.mark.parametrize("part,count", [("norm_forward_foldI", 33), ("norm_backward_foldI", 33), ("norm_forward_heldI", 12),
                                        ("norm_backward_heldI", 12), ("policy_heldI", 18), ("pref_gradientI", 15), ("dropout_kernelI", 12)])
def test_every_instance_is_looked_at(kernels, part, count):  # noqa: F811
    assert sum(part in name for name in kernels) == count
