"""Attention over caches in 4 bits (st_attn_*) at the ends of what its descriptors allow; formula, oracle and tolerances as in test_gpu_attn."""
import pytest

from paper_1901_00041_amd import st_conv as sc
from paper_1901_00041_amd import st_lm
from tests.attn_helpers import Tenant

pytestmark = pytest.mark.gpu


def torch_():
    import torch
    return torch


def run(t, opts=None, **changes):
    torch = torch_()
    plan = st_lm.st_attn_plan([t.upload().desc(**changes)], opts, keep=t)
    torch.cuda.synchronize()
    st_lm.st_attn_run(plan)
    torch.cuda.synchronize()
    return plan


# single tokens, a few, many rows, many rows whose tokens are divided, parts that are looked up; more new tokens than tokens among them
KINDS = [([(1, 700), (1, 1), (0, 9)], 0, None), ([(3, 259), (9, 4)], 0, None), ([(70, 133), (300, 300), (60, 20)], 1, None),
         ([(130, 1500), (70, 40), (1, 1)], 4, None), ([(40, 300), (2, 5)] + [(1, 30)] * 60, 2, 4096)]


@pytest.mark.parametrize("dim, dtype", [(64, "bf16"), (128, "f16"), (256, "bf16")])
@pytest.mark.parametrize("kind", range(len(KINDS)))
def test_a_window_as_long_as_the_table_hides_nothing(kind, dim, dtype):
    """Up to the largest number there is, which stands for no limit."""
    torch = torch_()
    seqs, split, max_new = KINDS[kind]
    t = Tenant(4, 2, dim, dtype, seqs, page=16, max_new=max_new)
    opts = sc.plan_opts(split_k=split)
    bad = st_lm.st_attn_status(run(t, opts))
    t.check_out("no window")
    whole = t.d["out"].clone()
    room = t.columns * t.page
    for window in (room, 1 << 30, 2 ** 31 - 257, 2 ** 31 - 1):
        plan = run(t, opts, window=window)
        t.check_out(f"window {window}")
        assert torch.equal(whole.view(torch.int16), t.d["out"].view(torch.int16)), window
        assert st_lm.st_attn_status(plan) == bad == (st_lm.ST_ATTN_BAD_LENGTH if any(n > length for n, length in seqs) else 0)
