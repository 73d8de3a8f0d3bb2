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


@pytest.mark.parametrize("what", ["type", "size", "count"])
def test_refused_gradients_change_nothing(what):
    """The first of the new ones is fit, of another type than the old; a later one is not."""
    given = lists(32)
    plan = Plan(**given)
    before = [t.grad for t in plan.tensors]
    seen = [weakref.ref(g) for g in given["grads"]]
    new = [torch.zeros(e) for e in SIZES]
    if what == "type":
        new[1] = new[1].bfloat16()
    elif what == "size":
        new[1] = new[1][:-1]
    else:
        new.pop()
    with pytest.raises(AssertionError):
        plan.set_grads(new)
    del given, new
    gc.collect()
    assert plan.grad_type == torch.bfloat16 and [t.grad for t in plan.tensors] == before
    assert [r().data_ptr() for r in seen] == before


def test_other_gradients_are_taken_and_held():
    plan = Plan(**lists(32))
    new = [torch.zeros(e) for e in SIZES]
    seen = [(weakref.ref(g), g.data_ptr()) for g in new]
    plan.set_grads(new)
    new.clear()
    gc.collect()
    assert plan.grad_type == torch.float32
    assert [(r().data_ptr(), t.grad) for (r, _), t in zip(seen, plan.tensors)] == [(a, a) for _, a in seen]


@pytest.mark.gpu
def test_a_step_after_refused_gradients():
    """It runs on the gradients that the plan had."""
    from helpers import ensure_built
    ensure_built()
    out = []
    for refuse in (False, True):
        p = [torch.ones(e, device="cuda").bfloat16() for e in SIZES]
        g = [torch.full((e,), 0.5, device="cuda").bfloat16() for e in SIZES]
        plan = oz.oz2_adamw_plan(p, g, **oz.oz2_adamw_states(p))
        if refuse:
            with pytest.raises(AssertionError):
                plan.set_grads([torch.full((SIZES[0],), -0.5, device="cuda"), torch.zeros(SIZES[1])])
        oz.oz2_adamw(plan, step=1, lr=1e-2)
        out.append(p)
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_masters_for_some_of_the_tensors():
    given = lists(32)
    given["masters"][0] = None
    plan = Plan(**given)
    assert plan.tensors[0].master is None
    assert plan.tensors[1].master == given["masters"][1].data_ptr()


@pytest.mark.gpu
def test_steps_with_masters_for_some():
    """A tensor's step does not depend on whether another has a master."""
    from helpers import ensure_built
    ensure_built()
    out = []
    for has in ((0, 0), (1, 1), (0, 1), (1, 0)):
        g = torch.Generator(device="cuda").manual_seed(3)
        p = [torch.randn(e, generator=g, device="cuda").bfloat16() for e in SIZES]
        grad = [torch.randn(e, generator=g, device="cuda").bfloat16() for e in SIZES]
        masters = [t.float() if h else None for t, h in zip(p, has)]
        plan = oz.oz2_adamw_plan(p, grad, masters=masters, **oz.oz2_adamw_states(p, bits=8))
        for step in (1, 2):
            oz.oz2_adamw(plan, step=step, lr=1e-2, seed=4)
        for t, m in zip(p, masters):
            assert m is None or torch.equal(t, m.bfloat16())
        out.append((p, masters))
    (none, _), (both, masters), (second, m2), (first, m1) = out
    assert torch.equal(second[0], none[0]) and torch.equal(first[1], none[1])
    assert torch.equal(second[1], both[1]) and torch.equal(m2[1], masters[1])
    assert torch.equal(first[0], both[0]) and torch.equal(m1[0], masters[0])
