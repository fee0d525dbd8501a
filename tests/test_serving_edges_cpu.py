"""Packed prompts and paged caches: what the host side does with a program's tensors and numbers, without a GPU."""
import paper_2412_03409_amd as P


def test_a_rotation_goes_by_where_the_plan_s_tensors_are():
    """Tensors whose storage is replaced: the old one may belong to somebody else by the next call."""
    plan, other = P.rope_plan(64, [16, 16], device="cpu"), P.rope_plan(32, [8, 8], theta=500.0, device="cpu")
    before = plan._args()
    assert plan._args() is before and before._obj.freq == plan.freq.data_ptr() and before._obj.rot_dim == 64
    plan.freq.data, plan.axis.data = other.freq.clone(), other.axis.clone()
    now = plan._args()._obj
    assert (now.freq, now.axis) == (plan.freq.data_ptr(), plan.axis.data_ptr())
    assert now.rot_dim == 32 and now.axes == 2
