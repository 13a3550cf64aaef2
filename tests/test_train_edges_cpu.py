"""What the operators around the graph layers refuse before they call anything, at its ends."""
import pytest

torch = pytest.importorskip("torch")


def test_steps_are_whole_numbers_whatever_came_before():
    from paper_2605_15695_amd.muon import Muon

    p = torch.nn.Parameter(torch.ones(2, 2))
    for steps in (5, 3):
        Muon([p], steps=steps)
        with pytest.raises(ValueError):
            Muon([p], steps=float(steps))
    opt = Muon([p])
    opt.param_groups[0]["steps"] = 5.0
    with pytest.raises(ValueError):
        opt.step()


@pytest.mark.parametrize("groups", [0, -4, 2.0, None])
def test_modules_of_no_groups_are_refused(groups):
    from paper_2605_15695_amd.norm import GroupNorm

    with pytest.raises(ValueError):
        GroupNorm(groups, 8)
