"""optim.AdamW refuses a step before anything of it has happened (CPU: as far as
that goes without a device)."""
import pytest
import torch

import paper_2305_17190_amd as pam
from paper_2305_17190_amd.optim import AdamW


def test_a_refused_first_step_makes_no_state():
    p = torch.nn.Parameter(torch.ones(3, 4))
    made = AdamW([p])
    p.grad = torch.ones(3, 4)
    with pytest.raises(pam.PamError, match="no CPU path"):
        made.step()
    assert not made.state and torch.equal(p, torch.ones(3, 4))


def test_types():
    p = torch.nn.Parameter(torch.ones(3, dtype=torch.bfloat16))
    made = AdamW([p])
    p.grad = torch.ones_like(p)
    with pytest.raises(TypeError, match="float32 parameters"):
        made.step()
    assert not made.state


@pytest.mark.parametrize("change", [dict(lr=float("nan")), dict(lr=-1.0), dict(eps=-1.0), dict(weight_decay=float("nan")),
                                    dict(betas=(0.9, 1.0))])
def test_rates_changed_to_none(change):
    """Of any group, before the first one steps."""
    a, b = (torch.nn.Parameter(torch.ones(3)) for _ in "ab")
    made = AdamW([dict(params=[a]), dict(params=[b])])
    a.grad, b.grad = torch.ones(3), torch.ones(3)
    made.param_groups[1].update(change)
    with pytest.raises(ValueError, match=next(iter(change))):
        made.step()
    assert not made.state
