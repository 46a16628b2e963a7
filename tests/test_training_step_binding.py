"""CPU: what the binding's AdamwPlan keeps alive, with the library's calls replaced by ones that note their arguments."""
import ctypes as C
import gc
import inspect
import os
import re
import struct
import weakref

import numpy as np
import pytest
import torch

from paper_1806_04090_amd import binding


class Library:
    """Stands for the library: every call succeeds and is noted; contexts and plans are numbers."""

    def __init__(self):
        self.calls, self.handles = [], 0

    def _create(self, name, args, out):
        self.handles += 1
        out._obj.value = self.handles
        self.calls.append((name, *args, self.handles))
        return 0

    def atomo_create(self, out, device):
        return self._create("create", (device,), out)

    def atomo_adamw_create(self, ctx, blob, n, out):
        if not ctx.value:
            return binding.ATOMO_EINVAL
        return self._create("adamw_create", (ctx.value, blob, n), out)

    def atomo_strerror(self, status):
        return b"an error"

    def atomo_adamw_destroy(self, ctx, plan):
        self.calls.append(("adamw_destroy", ctx.value, plan))
        return 0

    def atomo_destroy(self, ctx):
        self.calls.append(("destroy", ctx.value))
        return 0


@pytest.fixture
def library(monkeypatch):
    library = Library()
    monkeypatch.setattr(binding, "lib", lambda: library)
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    yield library
    gc.collect()                                                 # (whatever is left ends while the library is still replaced)


def context():
    ctx = binding.Context(0)
    ctx.index = -1                                               # what tensors in host memory give as their device
    return ctx


def eight_bit_model():
    """Lists for a plan, and the arrays whose memory its tensors have."""
    n = 300
    arrays = [np.ones(n, np.float32), np.ones(n, np.float16), *(np.zeros(k, np.uint8) for k in (n, n, 3, 3)), np.ones(n, np.float32)]
    p, g, m, v, m_scale, v_scale, copy = (torch.from_numpy(a) for a in arrays)
    return ([p], [g], [binding.AdamwState(m, v, m_scale, v_scale)], [copy]), arrays


def tensors_of(params, grads, states, copies):
    s = states[0]
    return [params[0], grads[0], s.m, s.v, s.m_scale, s.v_scale, copies[0]]


def addresses(library):
    """Those that the plan was made from: parameter, gradient, m, v, scales, copy."""
    (blob,) = [call[2] for call in library.calls if call[0] == "adamw_create"]
    return list(struct.unpack_from("7Q", blob, 8))


def clear_lists(params, grads, states, copies):
    for x in (params, grads, states, copies):
        x.clear()


def replace_in_lists(params, grads, states, copies):
    params[0], grads[0], copies[0], states[0] = torch.ones(1), torch.ones(1), torch.ones(1), binding.alloc_adamw_state(1, 32, "cpu")


def load_a_checkpoint(params, grads, states, copies):
    for name in ("m", "v", "m_scale", "v_scale"):
        setattr(states[0], name, getattr(states[0], name).clone())


def give_other_memory(params, grads, states, copies):
    for t in tensors_of(params, grads, states, copies):
        t.data = torch.zeros_like(t)


@pytest.mark.parametrize("change", [clear_lists, replace_in_lists, load_a_checkpoint, give_other_memory])
def test_a_plan_keeps_the_memory_that_it_was_made_from(library, change):
    ctx, (model, arrays) = context(), eight_bit_model()
    at, memory = [a.ctypes.data for a in arrays], [weakref.ref(a) for a in arrays]
    plan = binding.AdamwPlan(ctx, *model[:3], copies=model[3])
    assert addresses(library) == at
    del arrays
    change(*model)
    gc.collect()
    assert all(a() is not None for a in memory)
    plan.close()
    del model
    gc.collect()
    assert all(a() is None for a in memory)                      # and no longer than it has to


def names(library):
    return [(call[0], *call[-1:]) for call in library.calls]


def test_a_context_that_is_closed_closes_its_plans_first(library):
    ctx, other = context(), context()                            # handles 1 and 2
    (model, _), (second, _) = eight_bit_model(), eight_bit_model()
    plan, gone, theirs = binding.AdamwPlan(ctx, *model[:3]), binding.AdamwPlan(ctx, None, second[1]), binding.AdamwPlan(other, None, model[1])
    gone.close()
    ctx.close()
    assert names(library)[5:] == [("adamw_destroy", 4), ("adamw_destroy", 3), ("destroy", 1)]
    plan.close()                                                 # nothing is left to do
    ctx.close()
    assert len(library.calls) == 8
    with pytest.raises(binding.AtomoError):
        binding.AdamwPlan(ctx, None, second[1])
    theirs.close()
    other.close()
    assert names(library)[8:] == [("adamw_destroy", 5), ("destroy", 2)]


def test_plans_and_contexts_that_nothing_holds_any_more(library):
    ctx, (model, _) = context(), eight_bit_model()
    plan = binding.AdamwPlan(ctx, *model[:3])
    del ctx                                                      # the plan holds it
    gc.collect()
    assert len(library.calls) == 2
    del plan
    gc.collect()
    assert names(library)[2:] == [("adamw_destroy", 2), ("destroy", 1)]


def test_a_plan_and_its_context_in_one_piece_of_garbage(library):
    class Trainer:
        pass

    for plan_first in (False, True):
        t, (model, _), before = Trainer(), eight_bit_model(), len(library.calls)
        t.me, t.ctx = t, context()
        t.plan = binding.AdamwPlan(t.ctx, *model[:3])
        if plan_first:
            t.ctx.model = t
        del t
        gc.collect()
        ctx, plan = library.calls[before][-1], library.calls[before + 1][-1]
        assert names(library)[before + 2:] == [("adamw_destroy", plan), ("destroy", ctx)]


def test_the_seed_of_the_rounding_is_the_same_in_the_header_and_no_small_number(library):
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "atomo.h")).read()
    assert int(re.search(r"#define ATOMO_ADAMW_SEED (0x[0-9a-f]+)ull", text)[1], 16) == binding.ATOMO_ADAMW_SEED >= 2 ** 62
    assert inspect.signature(binding.atomo_adamw_step).parameters["seed"].default == binding.ATOMO_ADAMW_SEED
