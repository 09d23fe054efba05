"""Products of several tenants (st_matmul_*) without a GPU: what a plan refuses, and what it makes of the shapes it takes."""
import itertools

import pytest

from paper_1901_00041_amd import st_conv as sc
from paper_1901_00041_amd import st_lm

BASE = dict(M=4, N=16, K=32, in_dtype="bf16", out_dtype="bf16", x=0x100000, w=0x200000, y=0x300000)


def plan(*changes, **opts):
    return st_lm.st_matmul_plan([st_lm.make_matmul_desc(**{**BASE, **c}) for c in changes], sc.plan_opts(host_only=1, **opts))


@pytest.mark.parametrize("change, status", [
    (dict(M=-1), sc.ST_ERR_INVALID_ARG), (dict(N=0), sc.ST_ERR_INVALID_ARG), (dict(K=0), sc.ST_ERR_INVALID_ARG),
    (dict(in_dtype=7), sc.ST_ERR_UNSUPPORTED), (dict(out_dtype="f16"), sc.ST_ERR_UNSUPPORTED), (dict(in_dtype="f32", out_dtype="bf16"), sc.ST_ERR_UNSUPPORTED),
    (dict(epilogue=128), sc.ST_ERR_UNSUPPORTED), (dict(epilogue=st_lm.ST_EPI_RELU | st_lm.ST_EPI_GELU), sc.ST_ERR_INVALID_ARG),
    (dict(epilogue=st_lm.ST_EPI_RESIDUAL | st_lm.ST_EPI_RESIDUAL_LAST, residual=0x400000), sc.ST_ERR_INVALID_ARG),
    (dict(epilogue=st_lm.ST_EPI_BIAS), sc.ST_ERR_INVALID_ARG), (dict(epilogue=st_lm.ST_EPI_RESIDUAL), sc.ST_ERR_INVALID_ARG),
    (dict(x=None), sc.ST_ERR_INVALID_ARG), (dict(w=None), sc.ST_ERR_INVALID_ARG), (dict(y=None), sc.ST_ERR_INVALID_ARG),
    (dict(ldx=31), sc.ST_ERR_INVALID_ARG), (dict(ldw=-32), sc.ST_ERR_INVALID_ARG), (dict(ldy=15), sc.ST_ERR_INVALID_ARG),
    (dict(ldr=15, epilogue=st_lm.ST_EPI_RESIDUAL, residual=0x400000), sc.ST_ERR_INVALID_ARG),
    (dict(ldx=(1 << 21) + 1), sc.ST_ERR_UNSUPPORTED), (dict(K=(1 << 20) + 1), sc.ST_ERR_UNSUPPORTED), (dict(N=(1 << 20) + 1), sc.ST_ERR_UNSUPPORTED),
    (dict(x=0x100001), sc.ST_ERR_INVALID_ARG), (dict(y=0x300002, out_dtype="f32"), sc.ST_ERR_INVALID_ARG),
    (dict(y=0x100000), sc.ST_ERR_INVALID_ARG), (dict(y=0x100000 + 4 * 32 * 2 - 2), sc.ST_ERR_INVALID_ARG), (dict(y=0x200000 - 2), sc.ST_ERR_INVALID_ARG),
    (dict(epilogue=st_lm.ST_EPI_BIAS, bias=0x300000 + 8), sc.ST_ERR_INVALID_ARG),
    (dict(epilogue=st_lm.ST_EPI_RESIDUAL, residual=0x300000 + 2), sc.ST_ERR_INVALID_ARG),
    (dict(epilogue=st_lm.ST_EPI_RESIDUAL, residual=0x300000, ldr=20), sc.ST_ERR_INVALID_ARG),      # y itself, but not row for row
])
def test_refused(change, status):
    with pytest.raises(sc.StError) as refused:
        plan({}, change)
    assert refused.value.status == status


@pytest.mark.parametrize("change", [
    dict(epilogue=st_lm.ST_EPI_RESIDUAL_LAST, residual=0x300000),                          # in place
    dict(epilogue=st_lm.ST_EPI_RESIDUAL, residual=0x300000, ldr=24, ldy=24),
    dict(x=0x300000, ldx=48, y=0x300000 + 64, ldy=48),                                     # columns of one matrix
    dict(x=0x300000 + 32, ldx=48, y=0x300000, ldy=48),
    dict(x=0x300000 + 96 + 32, ldx=48, y=0x300000, ldy=48),                                # ... a row further down
    dict(y=0x100000 + 4 * 32 * 2), dict(x=0x100002), dict(M=0, x=None, w=None, y=None),
])
def test_accepted(change):
    assert st_lm.st_matmul_get_info(plan(change)).n_tenants == 1


def test_options_are_checked():
    for opts in (dict(tile_cfg=-1), dict(tile_cfg=st_lm.st_matmul_tile_count() + 1), dict(split_k=-1)):
        with pytest.raises(sc.StError) as refused:
            plan({}, **opts)
        assert refused.value.status == sc.ST_ERR_INVALID_ARG
    with pytest.raises(sc.StError):
        st_lm.st_matmul_tile_shape(st_lm.st_matmul_tile_count())
    with pytest.raises(sc.StError):
        st_lm.st_matmul_get_tenant_info(plan({}), 1)
    with pytest.raises(sc.StError) as refused:
        st_lm.st_matmul_run(plan({}))
    assert refused.value.status == sc.ST_ERR_UNSUPPORTED
    assert sc.lib().st_matmul_run(None, None) == sc.ST_ERR_INVALID_ARG


def test_empty_plans():
    info = st_lm.st_matmul_get_info(plan())
    assert (info.n_tenants, info.n_items, info.launches, info.flops, info.bytes) == (0, 0, 0, 0, 0)
    info = st_lm.st_matmul_get_info(plan(dict(M=0), dict(M=0, in_dtype="f32", out_dtype="f32")))
    assert (info.n_tenants, info.n_items, info.launches) == (2, 0, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_items_cover_the_outputs(dtype):
    sizes = [(1, 1, 1), (1, 4096, 4096), (7, 100, 33), (16, 17, 5000), (33, 64, 64), (65, 1000, 129), (129, 257, 8192), (300, 2000, 777), (4096, 8192, 4096)]
    p = plan(*[dict(M=m, N=n, K=k, in_dtype=dtype, out_dtype=dtype, x=1 << 40, w=2 << 40, y=3 << 40) for m, n, k in sizes])
    total = 0
    for t, (m, n, k) in enumerate(sizes):
        ti = st_lm.st_matmul_get_tenant_info(p, t)
        assert (ti.MT, ti.NT) == st_lm.st_matmul_tile_shape(ti.tile_cfg)
        assert (ti.tiles_m, ti.tiles_n) == (-(-m // ti.MT), -(-n // ti.NT))
        assert ti.split_k >= 1 and ti.item_count == ti.tiles_m * ti.tiles_n * ti.split_k
        total += ti.item_count
    info = st_lm.st_matmul_get_info(p)
    assert info.n_items == total and info.flops == sum(2 * m * n * k for m, n, k in sizes)
    es = 4 if dtype == "f32" else 2
    assert info.bytes == sum((m * k + n * k + m * n) * es for m, n, k in sizes)


def test_every_shape_and_division_can_be_asked_for():
    for cfg, split in itertools.product(range(st_lm.st_matmul_tile_count()), (1, 2, 5, 1000)):
        ti = st_lm.st_matmul_get_tenant_info(plan(dict(M=70, N=90, K=1000, x=1 << 40, w=2 << 40), tile_cfg=cfg + 1, split_k=split), 0)
        assert ti.tile_cfg == cfg and 1 <= ti.split_k <= split
        # slices of equally many steps: as many as asked for, or fewer where the last ones would be empty
        assert split < 2 or ti.split_k >= 2


def test_rebinding_is_checked():
    p = plan(dict(epilogue=st_lm.ST_EPI_BIAS, bias=0x500000))
    ok = st_lm.make_matmul_desc(**{**BASE, "bias": 0x600000})
    st_lm.st_matmul_rebind_all(p, [ok])
    for bad in (dict(x=None), dict(bias=None), dict(y=0x100000, bias=0x500000), dict(y=0x300001, bias=0x500000)):
        with pytest.raises(sc.StError) as refused:
            st_lm.st_matmul_rebind_all(p, [st_lm.make_matmul_desc(**{**BASE, **bad})])
        assert refused.value.status == sc.ST_ERR_INVALID_ARG
    with pytest.raises(sc.StError):
        st_lm.st_matmul_rebind_all(p, [ok, ok])
