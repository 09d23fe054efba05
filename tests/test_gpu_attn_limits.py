"""Attention over caches in 4 bits (st_attn_*) at the ends of what its descriptors allow; formula, oracle and tolerances as in test_gpu_attn."""
import numpy as np
import pytest

from paper_1901_00041_amd import st_conv as sc
from paper_1901_00041_amd import st_lm
from tests.attn_helpers import Tenant, attend, decode

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


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_what_the_cache_gives_back_of_every_value(dim, dtype):
    """All bit patterns of the type, by value: the elements that were written, each in the type, none beyond its largest number."""
    torch = torch_()
    heads = 4096 // dim
    t = Tenant(heads, heads, dim, dtype, [(16, 16)], page=16, filled=False)
    every = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(t.tt).double().numpy()
    finite = every[np.isfinite(every)]
    t.k[0] = np.concatenate([finite, np.zeros(65536 - finite.size)]).reshape(t.k[0].shape)
    t.v[0] = np.random.default_rng(7).permutation(t.k[0].ravel()).reshape(t.k[0].shape)      # large and small ones in one group
    plan = st_lm.st_attn_plan([t.upload().desc()], keep=t)
    st_lm.st_attn_append(plan)
    st_lm.st_attn_read(plan)
    torch.cuda.synchronize()
    t.fill([16])
    assert np.array_equal(t.d["pages"].cpu().numpy(), t.pool.bytes)
    most = torch.finfo(t.tt).max
    for name, held in zip(("k_out", "v_out"), t.held(0)):
        want = torch.from_numpy(held.transpose(1, 0, 2)).clamp(-most, most).to(t.tt).double().numpy()
        assert np.array_equal(t.outputs(name)[:16], want), name


@pytest.mark.parametrize("seqs, split", [([(1, 90)], 0), ([(3, 300)], 0), ([(80, 200)], 1), ([(70, 900)], 4)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_large_fp16_values_keep_their_size(dim, seqs, split):
    """Groups with a largest value above 49152, whose scale is 2^14: attention takes what the cache holds, 65536 among it."""
    t = Tenant(4, 2, dim, "f16", seqs, page=16, filled=False, gain=1e-3)
    rounded = lambda x: torch_().from_numpy(x).half().double().numpy()  # noqa: E731
    for x in (t.k[0], t.v[0]):
        x[:, :, ::32] = rounded(np.where(np.arange(x.shape[0])[:, None, None] % 2, 60000.0, -50000.0) + 0 * x[:, :, ::32])
        x[:, :, 1::32] = 30000.0
        x[:, :, 2::32] = -8192.0
    t.fill([seqs[0][1]])
    assert (t.held(0)[1] == 65536.0).any() and (t.held(0)[1] == 32768.0).any()
    run(t, sc.plan_opts(split_k=split))
    t.check_out()


@pytest.mark.parametrize("seqs, split", [([(1, 1), (1, 40)], 0), ([(3, 3), (2, 50)], 0), ([(80, 200)], 1), ([(70, 900)], 4)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_fp16_outputs_end_at_the_largest_number(dim, seqs, split):
    """Where all values are 60000, which the cache holds as 65536, and for keys of them that are not numbers."""
    t = Tenant(4, 2, dim, "f16", seqs, page=16, filled=False)
    for x in t.v:
        x[:], x[:, 1] = 60000.0, -65504.0
    t.k[-1][-1, 1, 5] = np.nan
    t.fill([length for _, length in seqs])
    run(t, sc.plan_opts(split_k=split))
    want = np.full(t.outputs().shape, np.nan)
    want[:t.first[-1], :2], want[:t.first[-1], 2:] = 65504.0, -65504.0
    want[t.first[-1] - 1, 2:] = np.nan             # the last token sees itself
    assert np.array_equal(t.outputs(), want, equal_nan=True)


@pytest.mark.parametrize("seqs", [[(1, 1)], [(80, 80)]])
def test_the_smallest_fp16_values(seqs):
    """Elements below 2^-22 may become multiples of 2^-23, half of which is 2^-24; the others are as they were, and the outputs' own rounding
    is of half a step, 2^-25, at most.  Every query sees tokens of the same values only."""
    t = Tenant(2, 1, 64, "f16", seqs, page=16, filled=False)
    t.v[0][:] = np.arange(64) * 2.0 ** -24
    t.fill([seqs[0][1]])
    run(t, sc.plan_opts(split_k=1))
    off = np.abs(t.outputs()[:seqs[0][0]] - t.held(0)[1][0, 0])
    assert off.max() <= 2.0 ** -24 + 2.0 ** -25 and off[..., 32:].max() <= 2.0 ** -25


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_every_scale_that_a_page_can_hold(dim, dtype):
    """Also those that only another type writes: an element that the type has no number for is rounded to one, or is its largest."""
    torch = torch_()
    t = Tenant(1, 1, dim, dtype, [(254, 254)], page=256, filled=False)
    code = np.tile(np.arange(16, dtype=np.uint8), dim // 16)[None]
    for p in range(254):
        scale = np.full((1, dim // 32), p + 1, np.uint8)
        t.pool.write(t.table[0, 0], p, code, scale, code[:, ::-1], scale)
    plan = st_lm.st_attn_plan([t.upload().desc()], keep=t)
    st_lm.st_attn_read(plan)
    torch.cuda.synchronize()
    most = torch.finfo(t.tt).max
    scale = np.minimum(np.arange(1, 255), 252)[:, None].repeat(dim // 32, 1)      # 2^125: the largest that anybody writes
    for name, codes in (("k_out", code), ("v_out", code[:, ::-1])):
        want = torch.from_numpy(decode(codes.repeat(254, 0), scale)).clamp(-most, most).to(t.tt).double().numpy()
        assert np.array_equal(t.outputs(name)[:254, 0], want), name


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("seqs, split, max_new", [([(5, 1), (1, 0), (7, 3)], 0, None), ([(40, 20), (70, 70), (90, 1)], 1, None), ([(300, 40), (64, 0)], 1, None),
                                                  ([(700, 600), (130, 1500), (300, 1)], 4, None), ([(60, 20), (2, 1)] + [(1, 30)] * 60, 1, 4096)])
def test_new_tokens_before_a_sequences_start_see_nothing(seqs, split, max_new, dim, dtype):
    """Without a causal mask, too: they get zeros, and the others see every token that there is."""
    t = Tenant(4, 2, dim, dtype, seqs, page=16, causal=False, max_new=max_new)
    plan = run(t, sc.plan_opts(split_k=split))
    got = t.outputs()
    for s, (n, length) in enumerate(seqs):
        before = max(0, n - length)
        mine = got[t.first[s]:t.first[s] + n]
        assert np.array_equal(mine[:before], np.zeros_like(mine[:before])), f"sequence {s}"
        if n > before:
            want, tol = attend(t.q[t.first[s] + before:t.first[s] + n], *t.held(s), length - (n - before), t.scale, False, 0, t.bits)
            assert (np.abs(mine[before:] - want) <= tol).all(), f"sequence {s}"
    t.check_untouched("", "out")
    assert st_lm.st_attn_status(plan) == st_lm.ST_ATTN_BAD_LENGTH


def test_rebinding_that_was_captured():
    """A graph that rebinds does so whenever it is replayed: the plan's own idea of the pointers does not make a later call do nothing."""
    torch = torch_()
    tenants = [Tenant(4, 2, 64, "bf16", [(1, 70), (1, 33)], page=16, seed=s).upload() for s in (1, 2)]
    a, b = tenants
    plan = st_lm.st_attn_plan([a.desc()], keep=tenants)
    x, w = torch.randn(2, 3, 64, device="cuda").unbind(0), torch.randn(40, 64, device="cuda")
    y = [torch.full((3, 40), float("nan"), device="cuda") for _ in range(2)]
    products = [st_lm.make_matmul_desc(3, 40, 64, "f32", "f32", x[i], w, y[i]) for i in range(2)]
    product = st_lm.st_matmul_plan([products[0]], keep=[x, w, y])
    side, graphs = torch.cuda.Stream(), [torch.cuda.CUDAGraph() for _ in range(2)]

    def step(which):
        st_lm.st_attn_rebind_all(plan, [tenants[which].desc()], side)
        st_lm.st_attn_run(plan, side)
        st_lm.st_matmul_rebind_all(product, [products[which]], side)
        st_lm.st_matmul_run(product, side)

    torch.cuda.synchronize()
    for which in range(2):         # the first one's pointers are the plan's own already
        with torch.cuda.graph(graphs[which], stream=side):
            step(which)
    want = [(x[i].double() @ w.double().t().contiguous()).cpu() for i in range(2)]
    tol = [2 * 2.0 ** -24 * 68 * (x[i].double().abs() @ w.double().abs().t().contiguous()).cpu() + 1e-30 for i in range(2)]

    def check(which, what):
        torch.cuda.synchronize()
        for i, t in enumerate(tenants):
            if i == which:
                t.check_out(what)
                assert ((y[i].double().cpu() - want[i]).abs() <= tol[i]).all(), what
            else:
                assert torch.isnan(t.d["out"]).all() and torch.isnan(y[i]).all(), what
        for t, z in zip(tenants, y):
            t.d["out"].fill_(float("nan"))
            z.fill_(float("nan"))
        torch.cuda.synchronize()

    step(1)                        # no graph has run yet
    check(1, "after the captures")
    for turn in range(3):
        for eager, replayed in ((0, 1), (1, 0), (0, 0)):
            step(eager)
            check(eager, f"eager {eager}, turn {turn}")
            graphs[replayed].replay()
            check(replayed, f"replay {replayed}, turn {turn}")
            step(eager)            # the pointers of the last eager call, but not always those that the replay left
            check(eager, f"eager {eager} again, turn {turn}")


@pytest.mark.parametrize("max_new", [None, 4096])
@pytest.mark.parametrize("dim, dtype", [(64, "bf16"), (64, "f16"), (128, "f16"), (256, "f16"), (256, "bf16")])
def test_attention_under_every_scale(dim, dtype, max_new):
    """Sequences of one token, whose value comes out as it is: scales above the largest one that the type writes count as that, the smallest elements are rounded."""
    torch = torch_()
    t = Tenant(2, 1, dim, dtype, [(1, 1)] * 255, page=16, filled=False, max_new=max_new)
    code = np.tile(np.arange(16, dtype=np.uint8), dim // 16)[None]
    zero, one = np.zeros((1, dim), np.uint8), np.ones((1, dim // 32), np.uint8)
    for p in range(255):
        t.pool.write(t.table[p, 0], 0, zero, one, code, p * one)
    run(t)
    largest = 141 if dtype == "f16" else 252          # 2^14, 2^125
    want = decode(code.repeat(255, 0), np.minimum(np.arange(255), largest)[:, None].repeat(dim // 32, 1))
    most = float(torch.finfo(t.tt).max)
    want = np.clip(want, -most, most)[:, None].repeat(2, 1)
    # fp16: multiples of 2^-23, then of 2^-24; bf16: what is below the smallest normal number may be 0
    off = np.abs(t.outputs()[:255] - want)
    assert (off <= (np.abs(want) < 2.0 ** -22) * (2.0 ** -24 + 2.0 ** -25) if dtype == "f16" else off <= (np.abs(want) < 2.0 ** -126) * 2.0 ** -126).all()
