"""Attention over caches in 4 bits (st_attn_*) without a GPU: refusals, page sizes, plans, and the oracle of the cache's elements."""
import numpy as np
import pytest

from paper_1901_00041_amd import st_conv as sc
from paper_1901_00041_amd import st_lm
from tests import attn_helpers as ah

POINTERS = dict(q=0x10000000, k=0x20000000, v=0x30000000, out=0x40000000, k_out=0x50000000, v_out=0x60000000, pages=0x70000000, table=0x1000, first=0x2000, length=0x3000)
BASE = dict(heads=8, kv_heads=2, head_dim=128, dtype="bf16", n_seqs=3, max_tokens=9, max_new=4, n_pages=20, page_tokens=32, table_pages=5, scale=0.1, flags=1, **POINTERS)


def plan(*changes, **opts):
    return st_lm.st_attn_plan([st_lm.make_attn_desc(**{**BASE, **c}) for c in changes], sc.plan_opts(host_only=1, **opts))


@pytest.mark.parametrize("change, status", [
    (dict(heads=0), sc.ST_ERR_INVALID_ARG), (dict(kv_heads=0), sc.ST_ERR_INVALID_ARG), (dict(heads=9), sc.ST_ERR_INVALID_ARG),
    (dict(head_dim=96), sc.ST_ERR_UNSUPPORTED), (dict(dtype="f32"), sc.ST_ERR_UNSUPPORTED),
    (dict(page_tokens=8), sc.ST_ERR_UNSUPPORTED), (dict(page_tokens=48), sc.ST_ERR_UNSUPPORTED), (dict(page_tokens=2048), sc.ST_ERR_UNSUPPORTED),
    (dict(n_seqs=-1), sc.ST_ERR_INVALID_ARG), (dict(max_tokens=-1), sc.ST_ERR_INVALID_ARG), (dict(max_new=0), sc.ST_ERR_INVALID_ARG),
    (dict(n_pages=-1), sc.ST_ERR_INVALID_ARG), (dict(table_pages=0), sc.ST_ERR_INVALID_ARG), (dict(window=-1), sc.ST_ERR_INVALID_ARG),
    (dict(window=5, flags=0), sc.ST_ERR_INVALID_ARG), (dict(flags=2), sc.ST_ERR_UNSUPPORTED),
    (dict(scale=float("nan")), sc.ST_ERR_INVALID_ARG), (dict(scale=float("inf")), sc.ST_ERR_INVALID_ARG),
    (dict(ldq=1023), sc.ST_ERR_INVALID_ARG), (dict(ldo=-1), sc.ST_ERR_INVALID_ARG), (dict(ldk=255), sc.ST_ERR_INVALID_ARG), (dict(ldv=255), sc.ST_ERR_INVALID_ARG),
    (dict(table_pages=1 << 26), sc.ST_ERR_UNSUPPORTED), (dict(max_new=1 << 29), sc.ST_ERR_UNSUPPORTED), (dict(heads=1 << 17), sc.ST_ERR_UNSUPPORTED),
    (dict(pages=0x70000008), sc.ST_ERR_INVALID_ARG), (dict(q=0x10000001), sc.ST_ERR_INVALID_ARG), (dict(table=0x1002), sc.ST_ERR_INVALID_ARG),
    (dict(out=0x10000000 + 512), sc.ST_ERR_INVALID_ARG), (dict(out=0x70000000 + 16), sc.ST_ERR_INVALID_ARG), (dict(k_out=0x60000000), sc.ST_ERR_INVALID_ARG),
    (dict(v_out=0x70000000), sc.ST_ERR_INVALID_ARG),
])
def test_refused(change, status):
    with pytest.raises(sc.StError) as refused:
        plan({}, change)
    assert refused.value.status == status


def test_reserved_and_null_arguments():
    d = st_lm.make_attn_desc(**BASE)
    d.reserved = 1
    with pytest.raises(sc.StError):
        st_lm.st_attn_plan([d], sc.plan_opts(host_only=1))
    L = st_lm.lib()
    assert L.st_attn_plan(None, 1, None, None) == sc.ST_ERR_INVALID_ARG
    assert L.st_attn_run(None, None) == L.st_attn_append(None, None) == L.st_attn_read(None, None) == sc.ST_ERR_INVALID_ARG
    assert L.st_attn_page_bytes(None) == -1
    with pytest.raises(sc.StError):
        plan({}, split_k=-1)
    p = plan({})
    for call in (st_lm.st_attn_run, st_lm.st_attn_append, st_lm.st_attn_read, st_lm.st_attn_status):
        with pytest.raises(sc.StError) as refused:
            call(p)
        assert refused.value.status == sc.ST_ERR_UNSUPPORTED
    L.st_attn_destroy(None)


def test_accepted_layouts():
    # queries, keys and values as columns of one matrix; in-place read-back; what is not needed is NULL
    row = (8 + 2 + 2) * 128
    plan(dict(q=0x10000000, k=0x10000000 + 8 * 256, v=0x10000000 + 10 * 256, ldq=row, ldk=row, ldv=row, k_out=0, v_out=0))
    plan(dict(k_out=0x20000000, v_out=0x30000000))
    plan({k: 0 for k in POINTERS})
    plan(dict(n_pages=0, pages=0))
    plan(dict(n_seqs=0, table_pages=0), dict(max_tokens=0), {})
    assert st_lm.st_attn_get_info(plan(dict(n_seqs=0, table_pages=0))).n_items == 0
    assert st_lm.st_attn_get_info(plan()).n_tenants == 0


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 64, 1024])
def test_page_bytes(dim, page):
    d = st_lm.make_attn_desc(**{**BASE, "head_dim": dim, "page_tokens": page})
    assert st_lm.st_attn_page_bytes(d) == ah.Pool(1, 2, page, dim).bytes.nbytes == 2 * page * (dim + dim // 16)
    assert st_lm.st_attn_page_bytes(st_lm.make_attn_desc(**{**BASE, "head_dim": dim, "page_tokens": page + 1})) < 0


def test_plans_divide_long_lengths():
    long = dict(n_seqs=1, max_new=1, max_tokens=1, table_pages=4096)
    assert st_lm.st_attn_get_info(plan(long)).n_items > 2 and st_lm.st_attn_get_info(plan(long)).workspace_bytes > 0
    assert st_lm.st_attn_get_info(plan(dict(long, window=100))).n_items == 2          # a window is short
    assert st_lm.st_attn_get_info(plan(long, split_k=1)).workspace_bytes == 0
    many = dict(long, max_new=500, max_tokens=500)
    assert st_lm.st_attn_get_info(plan(many)).workspace_bytes > 0                      # many rows, but few beside the chip
    assert st_lm.st_attn_get_info(plan(dict(many, n_seqs=100, max_tokens=50000))).workspace_bytes == 0
    both = st_lm.st_attn_get_info(plan(long, dict(long, dtype="f16"), dict(long, head_dim=64, ldq=0)))
    assert both.launches == 3


def test_rebinding_is_checked():
    p = plan({})
    st_lm.st_attn_rebind_all(p, [st_lm.make_attn_desc(**{**BASE, "q": 0x90000000})])
    for bad in (dict(pages=0x70000001), dict(out=0x10000000), dict(first=0x2001)):
        with pytest.raises(sc.StError):
            st_lm.st_attn_rebind_all(p, [st_lm.make_attn_desc(**{**BASE, **bad})])
    with pytest.raises(sc.StError):
        st_lm.st_attn_rebind_all(p, [])


def test_oracle_elements():
    """The oracle's own rule against the definition, value by value: scale from the mantissa of the largest, ties to even codes."""
    rng = np.random.default_rng(3)
    x = rng.standard_normal((50, 64)) * np.exp2(rng.integers(-30, 30, (50, 1)).astype(float))
    x[0] = 0.0
    x[1, :8] = [6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25]       # ties, with the scale 1 for a largest value of 6
    x[1, 8:] = 0.0
    code, scale = ah.encode(x)
    assert scale[1, 0] == 127 and scale[1, 1] == 1 and list(code[1, :8]) == [7, 6, 6, 4, 4, 2, 2, 0]
    held = ah.decode(code, scale)
    step = np.exp2(scale.astype(float) - 127).repeat(32, -1)
    assert (np.abs(held - x) <= step).all() and (np.abs(held - x)[np.abs(x) <= 2 * step] <= 0.25 * step[np.abs(x) <= 2 * step]).all()
    most = np.abs(x).reshape(50, -1, 32).max(-1)
    f = np.exp2(scale.astype(float) - 127)
    assert ((most <= 6 * f) & ((most > 3 * f) | (most == 0) | (scale == 1))).all()
    k = x.copy()
    k[2, 5], k[3, 40] = np.inf, np.nan
    kc, ks, vc, vs = ah.encode_token_head(k, x)
    assert (ks[2:4] == 255).all() and (vs[2:4] == 1).all() and not kc[2:4].any() and not vc[2:4].any() and (ks[4:] < 255).all()


def test_workgroups_follow_the_rows_that_there_can_be():
    """max_new = max_tokens: the sequences together have no more rows than that."""
    many = dict(n_seqs=1000, max_new=8192, max_tokens=8192, table_pages=256)
    # 192 rows of a key head's four query heads to a workgroup, one more for what a sequence leaves of one, and one that looks at the numbers
    assert st_lm.st_attn_get_info(plan(many)).n_items == 2 * (8192 * 4 // 192 + 1000) + 1
    assert st_lm.st_attn_get_info(plan(dict(many, n_seqs=1), split_k=1)).n_items == 2 * -(-8192 * 4 // 192)


def test_more_is_refused():
    far = 1 << 40
    for change, status in ((dict(k=0x70000000), sc.ST_ERR_INVALID_ARG), (dict(v=0x70000000 + 64), sc.ST_ERR_INVALID_ARG),
                           (dict(n_seqs=1 << 20, max_new=1, kv_heads=8, out=far), sc.ST_ERR_UNSUPPORTED)):
        with pytest.raises(sc.StError) as refused:
            plan(change)
        assert refused.value.status == status
