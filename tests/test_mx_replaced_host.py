"""A microscaled matrix whose tensors are replaced or take another shape, on the CPU: what the binding notices in Python."""
import pytest
import torch

from paper_2412_21124_amd import binding as B


class OnDevice(torch.Tensor):
    """A host tensor that says it is on the device: nothing here looks at its bytes."""
    device = property(lambda self: torch.device("cuda:0"))


def bytes_(*shape):
    return torch.zeros(*shape, dtype=torch.uint8).as_subclass(OnDevice)


def square():
    return B.MxTensor(bytes_(32, 32), bytes_(32, 32), 32, B.NT_MX_E4M3)


@pytest.mark.parametrize("name,value", [("codes", bytes_(32, 32)), ("scales", bytes_(32, 32)), ("rows", 16), ("cols", 16), ("format", B.NT_MX_E2M1),
                                        ("native", None), ("device", torch.device("cuda:1"))])
def test_attributes_are_not_assigned(name, value):
    m = square()
    before = getattr(m, name)
    with pytest.raises(AttributeError, match="make another"):
        setattr(m, name, value)
    assert getattr(m, name) is before
    m.pointer()


@pytest.mark.parametrize("which", ["codes", "scales"])
@pytest.mark.parametrize("change", [lambda t: t.t_(), lambda t: t.resize_(16, 32), lambda t: t.as_strided_((32, 16), (32, 1)), lambda t: t.set_(bytes_(32, 32)),
                                    lambda t: t.unsqueeze_(0)], ids=["turned", "fewer rows", "fewer columns", "other memory", "another dimension"])
def test_changed_in_place(which, change):
    m = square()
    change(getattr(m, which))
    with pytest.raises(RuntimeError, match="other memory or another shape"):
        m.pointer()


def test_other_attributes_are_the_programs_own():
    class Named(B.MxTensor):
        def __init__(self, name):
            super().__init__(bytes_(32, 32), bytes_(32, 32), 32, B.NT_MX_E4M3)
            self.name = name

    m = Named("up")
    m.name = m.step = "down"
    assert m.name == m.step == "down"
    with pytest.raises(AttributeError, match="make another"):
        m.scales = bytes_(32, 32)
