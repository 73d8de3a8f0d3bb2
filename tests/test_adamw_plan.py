"""What an AdamW plan holds: addresses of tensors, and so the tensors.  Its own Python
on CPU tensors (nothing is launched)."""
import gc
import weakref

import pytest
import torch

import paper_2606_06510_gb300 as oz

SIZES = (300, 7)


class Plan(oz.AdamWPlan):
    def _flat(self, t, numel, dtype, what):
        """As the plan's own check, of tensors anywhere."""
        assert t.dtype == dtype and t.numel() == numel and t.is_contiguous(), what
        return t.data_ptr() if numel else None


def lists(bits):
    """Every list that a plan takes."""
    p = [torch.zeros(e, dtype=torch.bfloat16) for e in SIZES]
    return {"params": p, "grads": [torch.zeros_like(t) for t in p], "masters": [t.float() for t in p],
            "m_scales": None, "v_scales": None, **oz.oz2_adamw_states(p, bits=bits), "lr_scales": None,
            "decay_scales": None}


FIELD = {"params": "param", "grads": "grad", "masters": "master", "m": "m", "v": "v", "m_scales": "m_scale",
         "v_scales": "v_scale"}


@pytest.mark.parametrize("bits", [32, 8])
def test_a_plan_holds_every_tensor_it_was_made_of(bits):
    """A caller's lists get other tensors (a checkpoint is loaded) or are cleared."""
    given = lists(bits)
    plan = Plan(**given)
    seen = {(name, i): (weakref.ref(t), t.data_ptr()) for name in FIELD for i, t in enumerate(given[name] or ())}
    for name in FIELD:
        if given[name]:
            given[name][0] = given[name][0].clone()
            given[name].clear()
    gc.collect()
    for (name, i), (ref, address) in seen.items():
        assert ref() is not None, (name, i)
        assert getattr(plan.tensors[i], FIELD[name]) == address == ref().data_ptr(), (name, i)
