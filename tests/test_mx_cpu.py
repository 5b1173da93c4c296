"""The 4-bit cache on the host: what its reference does to known numbers, and every refusal of its entry points (no GPU is touched:
the pointers are made up and nothing is launched)."""
import ctypes as C

import numpy as np
import pytest

import mx_reference as R
from paper_2601_23180_amd import binding as B
from test_abi_cpu import _model

ENULL, ESHAPE, ENODES, ETREE, ECAPACITY, EWORKSPACE, EARG, EMISMATCH = -1, -2, -3, -4, -6, -7, -8, -9


def desc(**kw):
    base = dict(k_codes=0x10000, k_scales=0x20000, v_codes=0x30000, v_scales=0x40000, page_table=None, batch=2, n_kv_heads=4,
                head_dim=128, capacity=512, max_pages=0, n_pages=0)
    base.update(kw)
    return B.MXCacheDesc(*[base[k] for k, _ in B.MXCacheDesc._fields_])


def ints(*v):
    return (C.c_int32 * len(v))(*v)


def rows(data=0x50000, row=512, seq=512 * 16):
    return B.MXRows(data, row, seq)


def test_reference_rounds_to_the_format():
    x = np.zeros((1, 32))
    x[0, :12] = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.26, 0.74, 1e-9, -5.01]
    code, byte = R.quantise(x)
    assert byte[0, 0] == 127
    want = [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -0.5, 0.5, 0.0, -6.0]
    np.testing.assert_array_equal(R.values(code, byte)[0, :12], want)
    for top, e in ((6.99, 127), (7.0, 128), (4.0, 127), (3.99, 127), (3.5, 127), (3.49, 126), (2.0 ** -126, 0), (1e-45, 0), (3.4e38, 252)):
        assert R.quantise(np.full((1, 32), top))[1][0, 0] == e, top
    assert R.quantise(np.zeros((1, 32)))[1][0, 0] == 0
    x[0, 5] = np.inf
    assert R.quantise(x)[1][0, 0] == 255 and np.isnan(R.rounded(x)).all()


def test_sizes():
    lib, a, b = B.lib(), C.c_size_t(), C.c_size_t()
    assert lib.trispec_mx_cache_bytes(C.byref(desc()), C.byref(a), C.byref(b)) == 0
    assert a.value == 2 * 4 * 512 * 64 and b.value == 2 * 4 * 512 * 4
    paged = desc(page_table=0x60000, max_pages=3, n_pages=7, head_dim=64, capacity=0)
    assert lib.trispec_mx_cache_bytes(C.byref(paged), C.byref(a), C.byref(b)) == 0
    assert a.value == 7 * 4 * 256 * 32 and b.value == 7 * 4 * 256 * 2
    for bad, rc in ((desc(batch=0), ENODES), (desc(batch=9), ENODES), (desc(head_dim=96), ESHAPE), (desc(n_kv_heads=0), ESHAPE),
                    (desc(capacity=100), ECAPACITY), (desc(capacity=0), ECAPACITY),
                    (desc(page_table=0x60000, max_pages=0, n_pages=1), ECAPACITY), (desc(page_table=0x60000, max_pages=1, n_pages=0), ECAPACITY)):
        assert lib.trispec_mx_cache_bytes(C.byref(bad), C.byref(a), C.byref(b)) == rc
    assert lib.trispec_mx_cache_bytes(None, C.byref(a), C.byref(b)) == ENULL
    assert lib.trispec_mx_cache_bytes(C.byref(desc()), None, C.byref(b)) == ENULL
    assert lib.trispec_mx_attend_workspace_bytes(1, 1, 32, 8, 128, C.byref(a)) == 0 and a.value > 0
    for bad, rc in (((0, 1, 32, 8, 128), ENODES), ((1, 129, 8, 8, 128), ENODES), ((8, 64, 8, 8, 128), ENODES), ((1, 1, 30, 8, 128), ESHAPE),
                    ((1, 1, 72, 8, 128), ESHAPE), ((1, 1, 32, 8, 96), ESHAPE), ((1, 65, 64, 8, 128), ENODES)):
        assert lib.trispec_mx_attend_workspace_bytes(*bad, C.byref(a)) == rc, bad


@pytest.mark.parametrize("which", ["append", "read"])
def test_rows_are_checked_before_any_launch(which):
    fn = B.lib().trispec_mx_append if which == "append" else B.lib().trispec_mx_read

    def call(c=None, k=None, v=None, dtype=1, start=ints(0, 0), count=ints(4, 4)):
        c, k, v = c or desc(), k or rows(), v or rows()
        return fn(C.byref(c), C.byref(k), C.byref(v), dtype, start, count, None)

    assert fn(None, C.byref(rows()), C.byref(rows()), 1, ints(0, 0), ints(1, 1), None) == ENULL
    assert call(k=rows(data=None)) == ENULL and call(v=rows(data=None)) == ENULL
    assert call(c=desc(v_scales=None)) == ENULL and call(c=desc(k_codes=0x10008)) == EARG
    assert call(start=None) == ENULL and call(count=None) == ENULL
    assert call(dtype=2) == EARG
    assert call(k=rows(data=0x50008)) == EARG and call(v=rows(row=516)) == EARG and call(k=rows(seq=4)) == EARG and call(k=rows(row=-512)) == EARG
    assert call(start=ints(-1, 0)) == ECAPACITY and call(count=ints(0, -1)) == ECAPACITY
    assert call(start=ints(0, 509)) == ECAPACITY and call(start=ints(2 ** 31 - 1, 0)) == ECAPACITY and call(count=ints(2 ** 31 - 1, 0)) == ECAPACITY
    assert call(c=desc(batch=0)) == ENODES
    assert call(c=desc(page_table=0x60002, max_pages=2, n_pages=4)) == EARG
    assert call(start=ints(512, 3), count=ints(0, 0)) == 0                       # nothing to do, nothing launched
    if which == "read":
        assert fn(C.byref(desc()), None, None, 1, ints(0, 0), ints(1, 1), None) == ENULL
        assert call(k=rows(row=256)) == EARG                                     # rows of 512 elements would overlap
        assert call(v=rows(seq=1024)) == EARG                                    # 4 rows of 512: sequences would overlap
        assert call(k=rows(row=0), count=ints(2, 0)) == EARG
    else:
        assert fn(C.byref(desc()), None, C.byref(rows()), 1, ints(0, 0), ints(1, 1), None) == ENULL


def test_attention_is_checked_before_any_launch():
    lib = B.lib()

    def call(c=None, ctx=ints(10, 20), tree_parents=None, **kw):
        c = c or desc()
        base = dict(q=rows(row=1024), k=rows(), v=rows(), dtype=1, n_nodes=3, n_q_heads=8, append=0, out=0x70000,
                    out_row_stride=1024, workspace=0x80000, workspace_bytes=1 << 40, stream=None)
        base.update(kw)
        a = B.MXAttendArgs(*[base[k] for k, _ in B.MXAttendArgs._fields_])
        return lib.trispec_mx_attend(C.byref(c), ctx, tree_parents, C.byref(a))

    none = B.MXRows(None, 0, 0)
    assert call(q=none) == ENULL and call(k=none) == ENULL and call(v=none) == ENULL and call(out=None) == ENULL and call(ctx=None) == ENULL
    assert call(k=none, v=none, append=1) == ENULL
    assert call(c=desc(k_codes=None)) == ENULL
    assert call(n_nodes=0) == ENODES and call(n_nodes=129) == ENODES and call(c=desc(batch=8), n_nodes=33, ctx=ints(*[0] * 8)) == ENODES
    assert call(n_q_heads=6) == ESHAPE and call(n_q_heads=36) == ESHAPE and call(n_q_heads=0) == ESHAPE
    assert call(n_nodes=65, n_q_heads=32, q=rows(row=4096), out_row_stride=4096) == ENODES          # 520 query rows a kv head
    assert call(dtype=3) == EARG and call(append=2) == EARG and call(out=0x70008) == EARG
    assert call(out_row_stride=1016) == EARG and call(out_row_stride=1028) == EARG and call(q=rows(row=1028)) == EARG
    assert call(ctx=ints(513, 0)) == ECAPACITY and call(ctx=ints(0, -1)) == ECAPACITY and call(ctx=ints(510, 0), append=1) == ECAPACITY
    for tree in ((0, 0, 1), (-1, 0, 2), (-1, -1, 0), (-1, 0, -2)):
        assert call(tree_parents=ints(-1, 0, 1, *tree)) == ETREE, tree
    assert call(workspace=None) == EWORKSPACE and call(workspace=0x80010) == EWORKSPACE and call(workspace_bytes=1024) == EWORKSPACE


def test_cache_object_is_checked():
    lib = B.lib()
    rc, m, keep = _model(dtype=B.TRISPEC_BF16, n_kv_heads=2, head_dim=64)
    assert rc == 0
    kv = C.c_void_p()
    ok = dict(n_kv_heads=2, head_dim=64, batch=1, capacity=256)
    assert lib.trispec_kv_create_mx(None, C.byref(desc(**ok)), C.byref(kv)) == ENULL
    assert lib.trispec_kv_create_mx(m, C.byref(desc(**ok)), None) == ENULL
    assert lib.trispec_kv_create_mx(m, C.byref(desc(**{**ok, "n_kv_heads": 4})), C.byref(kv)) == EMISMATCH
    assert lib.trispec_kv_create_mx(m, C.byref(desc(**{**ok, "head_dim": 128})), C.byref(kv)) == EMISMATCH
    assert lib.trispec_kv_create_mx(m, C.byref(desc(**{**ok, "v_codes": 0x30004})), C.byref(kv)) == EARG
    assert lib.trispec_kv_create_mx(m, C.byref(desc(**ok)), C.byref(kv)) == 0
    assert lib.trispec_kv_set_len(kv, ints(257)) == ECAPACITY and lib.trispec_kv_set_len(kv, ints(250)) == 0
    lib.trispec_kv_destroy(kv)
    paged = desc(**{**ok, "page_table": 0x60000, "max_pages": 3, "n_pages": 5, "capacity": 0})
    assert lib.trispec_kv_create_mx(m, C.byref(paged), C.byref(kv)) == 0
    assert lib.trispec_kv_set_len(kv, ints(768)) == 0 and lib.trispec_kv_set_len(kv, ints(769)) == ECAPACITY
    lib.trispec_kv_destroy(kv)
    rc, f, keep_f = _model(n_kv_heads=2, head_dim=64)
    assert lib.trispec_kv_create_mx(f, C.byref(desc(**ok)), C.byref(kv)) == ESHAPE       # an fp32 model keeps fp32
    lib.trispec_model_destroy(m)
    lib.trispec_model_destroy(f)
