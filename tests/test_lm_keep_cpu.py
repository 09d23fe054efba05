"""What plans of products and attention keep alive for their callers (st_lm), without a GPU."""
import weakref

import pytest

from paper_1901_00041_amd import st_conv as sc
from paper_1901_00041_amd import st_lm


class Tensors:
    """Stands for a set of tensors; can be watched."""


def matmul(x):
    return st_lm.make_matmul_desc(4, 16, 32, "bf16", "bf16", 0x100000 + x, 0x200000, 0x300000)


def attn(x):
    return st_lm.make_attn_desc(8, 2, 128, "bf16", 3, 9, 4, 20, 32, 5, q=0x10000000 + x, out=0x40000000, pages=0x70000000, table=0x1000, first=0x2000, length=0x3000)


@pytest.mark.parametrize("make, plan_of, rebind", [(matmul, st_lm.st_matmul_plan, st_lm.st_matmul_rebind_all), (attn, st_lm.st_attn_plan, st_lm.st_attn_rebind_all)])
def test_what_a_plan_holds_is_let_go_when_its_caller_says_so(make, plan_of, rebind):
    sets = [Tensors() for _ in range(5)]
    seen = [weakref.ref(s) for s in sets]
    plan = plan_of([make(0)], sc.plan_opts(host_only=1), keep=sets[0])
    for turn in range(3):                     # a set that comes round again is held once
        for i, s in enumerate(sets):
            rebind(plan, [make(64 * i)], keep=s)
    assert len(plan.kept) == 5
    del sets, s
    assert all(r() is not None for r in seen)
    rebind(plan, [make(640)])                 # nothing new to hold: everything stays
    assert all(r() is not None for r in seen)
    plan.release(keep=seen[3]())
    assert [r() is not None for r in seen] == [False, False, False, True, False]
    plan.release()
    assert seen[3]() is None and plan.kept == []
    last = Tensors()
    gone = weakref.ref(last)
    rebind(plan, [make(0)], keep=last)
    del last
    assert gone() is not None
    plan.destroy()                            # which waits for the device
    assert gone() is None


def test_a_thousand_rebindings_nest_nothing():
    plan = st_lm.st_matmul_plan([matmul(0)], sc.plan_opts(host_only=1), keep=[])
    for i in range(1000):
        st_lm.st_matmul_rebind_all(plan, [matmul(64 * i)], keep=(i,))
        if i % 2:
            plan.release(keep=(i,))
    assert plan.kept == [(999,)]


def test_a_refused_rebinding_keeps_nothing():
    plan = st_lm.st_matmul_plan([matmul(0)], sc.plan_opts(host_only=1))
    refused = Tensors()
    seen = weakref.ref(refused)
    with pytest.raises(sc.StError):
        st_lm.st_matmul_rebind_all(plan, [st_lm.make_matmul_desc(4, 16, 32, "bf16", "bf16", None, None, None)], keep=refused)
    del refused
    assert seen() is None and plan.kept == []
