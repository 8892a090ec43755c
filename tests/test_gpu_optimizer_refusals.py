"""optim.AdamW: a refused step changes no parameter and no state, of no group, and
the next one goes on as if it had not been."""
import pytest

import paper_2305_17190_amd as pam
from gpu_util import device, note

pytestmark = pytest.mark.gpu


def parameters(seed=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return [torch.nn.Parameter(torch.randn(*s, generator=g).to(device())) for s in ((40, 30), (30,), (20, 300))]


def gradients(params, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    for p in params:
        p.grad = torch.randn(p.shape, generator=g).to(device())


# What is wrong, after so many steps: shared memory is looked for when states are
# made, a state has to be there to be a wrong one.
BREAKS = [(how, before) for how in ("transposed", "bfloat16", "cpu", "rate") for before in (0, 2)] + [("shared", 0),
                                                                                                     ("state", 2)]


@pytest.mark.parametrize("how,before", BREAKS)
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("max_norm", [None, 0.5])
def test_a_refused_step(how, bits, max_norm, before):
    import torch
    from paper_2305_17190_amd.optim import AdamW
    note(f"AdamW refused by {how}, {bits} bits, max_norm {max_norm}, after {before} steps")
    mine, other = parameters(), parameters()
    a, b = (AdamW([dict(params=x[:2]), dict(params=x[2:], lr=1e-2)], state_bits=bits, max_norm=max_norm, seed=2)
            for x in (mine, other))
    for step in range(before):
        for x, opt in ((mine, a), (other, b)):
            gradients(x, step)
            opt.step()
    gradients(mine, 10)
    last, good, grad = mine[2], mine[2].data, mine[2].grad
    if how == "transposed":
        last.data = good.t().contiguous().t()
    elif how == "bfloat16":
        last.grad = None
        last.data = good.bfloat16()
        last.grad = grad.bfloat16()
    elif how == "cpu":
        last.grad = None
        last.data = good.cpu()
        last.grad = grad.cpu()
    elif how == "shared":
        extra = torch.nn.Parameter(good[:3])
        extra.grad = torch.ones_like(extra)
        a.param_groups[1]["params"].append(extra)
    elif how == "rate":
        a.param_groups[1]["lr"] = float("nan")
    elif how == "state":
        kept = a.state[last]["sq"]
        a.state[last]["sq"] = kept.reshape(-1)[1:].clone()
    old = [p.detach().clone() for p in mine]
    states = {p: {k: v.clone() if torch.is_tensor(v) else v for k, v in s.items()} for p, s in a.state.items()}
    with pytest.raises((TypeError, ValueError, pam.PamError)):
        a.step()
    assert all(torch.equal(x, y) for x, y in zip(old, mine))
    assert set(states) == set(a.state)
    for p, s in a.state.items():
        assert s.keys() == states[p].keys()
        assert all(torch.equal(v, states[p][k]) if torch.is_tensor(v) else v == states[p][k] for k, v in s.items())
    # Mended, it steps as the other does.
    last.grad = None
    last.data = good
    last.grad = grad
    if how == "shared":
        a.param_groups[1]["params"].pop()
    elif how == "rate":
        a.param_groups[1]["lr"] = 1e-2
    elif how == "state":
        a.state[last]["sq"] = kept
    gradients(other, 10)
    a.step()
    b.step()
    assert all(torch.equal(x, y) for x, y in zip(mine, other))


def test_parameters_joining_later():
    """One whose gradient came first in the third step, beside others: as torch's."""
    import torch
    from paper_2305_17190_amd.optim import AdamW
    note("AdamW, a parameter joining later")
    mine, other = parameters(), parameters()
    a, b = AdamW(mine, lr=1e-3), torch.optim.AdamW(other, lr=1e-3)
    for step in range(6):
        for x, opt in ((mine, a), (other, b)):
            gradients(x, step)
            if step < 2:
                x[1].grad = None
            opt.step()
    assert [a.state[p]["step"] for p in mine] == [6, 4, 6]
    assert all(torch.allclose(x, y, rtol=1e-5, atol=1e-6) for x, y in zip(mine, other))
