"""CPU tests of the optimiser's bookkeeping: what copies and saved states carry."""
import copy
import pickle

import torch

from paper_2607_20652_gb300.optim import AdamW


def test_copies_and_saved_states_carry_the_seed():
    p = [torch.nn.Parameter(torch.zeros(4)), torch.nn.Parameter(torch.zeros(3))]
    opt = AdamW([{"params": p[:1]}, {"params": p[1:], "lr": 1e-4}], state_bits=8, seed=11)
    for other in (copy.deepcopy(opt), pickle.loads(pickle.dumps(opt))):
        assert other.seed == 11 and other._sets == {} and [g["seed"] for g in other.param_groups] == [11, 11]
        assert other.param_groups[0]["params"][0] is not p[0]
    saved = opt.state_dict()
    late = AdamW([{"params": p[:1]}, {"params": p[1:]}], state_bits=8)
    late.load_state_dict(saved)
    assert late.seed == 11
    for g in saved["param_groups"]:  # saved before seeds were kept there
        del g["seed"]
    late = AdamW([{"params": p[:1]}, {"params": p[1:]}], state_bits=8, seed=5)
    late.load_state_dict(saved)
    assert late.seed == 5
    late.seed = 6
    late.add_param_group({"params": [torch.nn.Parameter(torch.zeros(2))]})
    assert [g["seed"] for g in late.param_groups] == [6, 6, 6]


def test_a_step_without_gradients_needs_no_device():
    p = torch.nn.Parameter(torch.zeros(4))
    opt = AdamW([p])
    assert opt.step(lambda: 3.0) == 3.0 and not opt.state[p]
