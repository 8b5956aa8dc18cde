"""The paged-cache calls are exported as include/locks_cache.h declares them and refuse bad
arguments on the host before any launch; the binding checks tensors first (no GPU)."""
import ctypes
import os
import re

import pytest
import torch

from paper_2607_24555_amd import cache as C
from paper_2607_24555_amd import locks as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "locks_cache.h")
FAKE = ctypes.c_void_p(0x1000)
ODD = ctypes.c_void_p(0x1008)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return C.lib()


def cfg(**kw):
    c = B.Config(num_seqs=2, num_q_heads=8, num_kv_heads=2, rank=8, budget_tokens=256,
                 max_pages_per_seq=64, num_blocks=128)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rows(**kw):
    r = C._Rows(0x1000, 0x1000, 0x1000, 0x2000, 0x1000, 1024, 256, 256, 1024, 5)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def rope(pairs=(64, 0, 0), **kw):
    r = C._Rope(0x1000, None, 100, 128, 0, 1, (ctypes.c_int32 * 3)(*pairs))
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def q8(**kw):
    r = C._Q8(0x1000, 0x1000, 0x1000, 0x1000, 0)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def test_every_declared_symbol_is_exported(lib):
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(locks_[a-z_0-9]+)\s*\(", src))
    assert names == set(C._SIGS), "binding and header disagree"
    for n in names:
        assert hasattr(lib, n), n


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _rope_append(lib, c, r, p, kc=FAKE, vc=FAKE, pt=FAKE, sl=FAKE):
    return lib.locks_rope_append_kv(_ref(c), _ref(r), _ref(p), kc, vc, pt, sl, None)


def _q8_append(lib, c, r, p, store=q8(), pt=FAKE, sl=FAKE):
    return lib.locks_q8_append_kv(_ref(c), _ref(r), _ref(p), _ref(store), pt, sl, None)


def _appends(lib, c, r, p, **tables):
    """Both appends; only for arguments that both refuse (or that launch nothing)."""
    return _rope_append(lib, c, r, p, **tables), _q8_append(lib, c, r, p, **tables)


@pytest.mark.parametrize("bad,code", [
    (dict(k=None), -1), (dict(v=None), -1), (dict(k=0x1008), -1), (dict(v=0x1001), -1),
    (dict(q_out=None), -1), (dict(q_out=0x2004), -1), (dict(q=0x1002), -1), (dict(n_tokens=-1), -1),
    (dict(k_stride=255), -1), (dict(k_stride=260), -1), (dict(v_stride=0), -1), (dict(v_stride=-256), -1),
    (dict(q_stride=1020), -1), (dict(q_out_stride=512), -1), (dict(k_stride=1 << 41), -1),
    (dict(cu_tokens=None), -1),                    # five rows, two sequences
    (dict(q_out=0x1000, q_out_stride=2048), -1),   # in place with another stride
])
def test_bad_rows_are_rejected(lib, bad, code):
    assert _appends(lib, cfg().c(), rows(**bad), rope()) == (code, code)


@pytest.mark.parametrize("bad,code", [
    (dict(rot_dim=0), -2), (dict(rot_dim=8), -2), (dict(rot_dim=40), -2), (dict(rot_dim=144), -2),
    (dict(n_pos=0), -1), (dict(table=0x1004), -1), (dict(interleaved=2), -1), (dict(n_axes=0), -1),
    (dict(n_axes=4), -1), (dict(n_axes=2), -1), (dict(rot_dim=64), -1), (dict(pairs=(63, 1, 0)), -1),
    (dict(pairs=(70, -6, 0), n_axes=2, positions=0x1000), -1), (dict(pairs=(0, 0, 0)), -1),
])
def test_bad_rotations_are_rejected(lib, bad, code):
    assert _appends(lib, cfg().c(), rows(), rope(**bad)) == (code, code)


def test_null_arguments_and_empty_batches(lib):
    c = cfg().c()
    assert _appends(lib, None, rows(), rope()) == (-1, -1)
    assert _appends(lib, c, None, rope()) == (-1, -1)
    assert _appends(lib, c, rows(), rope(), pt=None) == (-1, -1)
    assert _appends(lib, c, rows(), rope(), sl=None) == (-1, -1)
    assert _rope_append(lib, c, rows(), rope(), kc=None) == -1
    assert _rope_append(lib, c, rows(), rope(), vc=ODD) == -1
    assert _q8_append(lib, c, rows(), rope(), store=None) == -1
    assert _appends(lib, cfg(head_dim=64).c(), rows(), rope()) == (-2, -2)
    assert _appends(lib, cfg(kv_dtype=5).c(), rows(), rope()) == (-2, -2)
    # nothing to append: no launch
    assert _appends(lib, c, rows(n_tokens=0), rope()) == (0, 0)
    assert _appends(lib, c, rows(n_tokens=0, k=None, v=None, q=None, q_out=None), None) == (0, 0)
    assert _appends(lib, cfg(num_seqs=0).c(), rows(n_tokens=0, cu_tokens=None), None) == (0, 0)
    # fp32 rows need strides of 16 bytes too
    f = cfg(kv_dtype=B.LOCKS_FP32, q_dtype=B.LOCKS_FP32).c()
    assert _appends(lib, f, rows(k_stride=258), rope()) == (-1, -1)


@pytest.mark.parametrize("bad,code", [(dict(code=2), -2), (dict(code=-1), -2), (dict(k=None), -1),
                                      (dict(v=None), -1), (dict(k_scale=None), -1),
                                      (dict(v_scale=None), -1), (dict(k=0x1008), -1), (dict(v=0x1004), -1)])
def test_bad_stores_are_rejected(lib, bad, code):
    c = cfg().c()
    need = lib.locks_workspace_bytes(ctypes.byref(c))
    s = q8(**bad)
    assert _q8_append(lib, c, rows(), rope(), s) == code
    assert lib.locks_q8_dense_attend(ctypes.byref(c), FAKE, ctypes.byref(s), FAKE, FAKE, FAKE, None, FAKE,
                                     need, None) == code
    assert lib.locks_q8_sparse_attend(ctypes.byref(c), FAKE, ctypes.byref(s), FAKE, FAKE, FAKE, FAKE, None,
                                      FAKE, need, None) == code


def test_build_arguments(lib):
    c, s = cfg().c(), q8()
    build = lambda c=c, s=s, pt=FAKE, sl=FAKE, lst=None, n=0, out=FAKE: lib.locks_q8_build_summaries(
        ctypes.byref(c), _ref(s), pt, sl, lst, n, out, None)
    assert build(s=None) == build(pt=None) == build(sl=None) == build(out=None) == -1
    assert build(n=-1) == build(n=3) == -1 and build(s=q8(code=9)) == -2 and build(s=q8(k=0x1001)) == -1
    assert build(c=cfg(rank=0).c()) == -1 and build(c=cfg(num_seqs=0).c()) == 0


def test_attention_arguments(lib):
    c, s = cfg().c(), q8()
    need = lib.locks_workspace_bytes(ctypes.byref(c))
    dense = lambda c=c, q=FAKE, s=s, pt=FAKE, sl=FAKE, out=FAKE, ws=FAKE, n=need: lib.locks_q8_dense_attend(
        ctypes.byref(c), q, None if s is None else ctypes.byref(s), pt, sl, out, None, ws, n, None)
    assert dense(q=None) == dense(q=ODD) == dense(s=None) == dense(pt=None) == dense(sl=None) == dense(out=None) == -1
    assert dense(out=ODD) == -1
    # 16 x 8 x 2^24 x 4 units
    wide = cfg(num_seqs=16, num_q_heads=8, num_kv_heads=8, max_pages_per_seq=1 << 24, page_size=64).c()
    assert dense(c=wide, n=1 << 62) == -2
    assert dense(ws=None) == dense(n=need - 1) == dense(ws=ctypes.c_void_p(0x1010)) == -3
    assert dense(c=cfg(page_size=48).c()) == -2 and dense(c=cfg(budget_tokens=1).c()) == -1
    assert lib.locks_q8_sparse_attend(ctypes.byref(c), FAKE, ctypes.byref(s), FAKE, FAKE, None, FAKE, None,
                                      FAKE, need, None) == -1
    z = cfg(num_seqs=0).c()
    assert dense(c=z, n=lib.locks_workspace_bytes(ctypes.byref(z))) == 0


def _tensors(n=2, dt=torch.bfloat16):
    c = cfg(num_blocks=6, max_pages_per_seq=3)
    return c, dict(k=torch.zeros(n, 2, 128, dtype=dt), v=torch.zeros(n, 2, 128, dtype=dt),
                   pt=torch.zeros(2, 3, dtype=torch.int32), sl=torch.zeros(2, dtype=torch.int32),
                   kc=torch.zeros(6, 2, 16, 128, dtype=dt), vc=torch.zeros(6, 2, 16, 128, dtype=dt))


@pytest.mark.parametrize("over,msg", [
    (dict(k=torch.zeros(2, 2, 128)), "k_new: dtype"),
    (dict(k=torch.zeros(3, 2, 128, dtype=torch.bfloat16)), "without cu_tokens"),
    (dict(k=torch.zeros(2, 256, dtype=torch.bfloat16)), "k_new: expected"),
    (dict(pt=torch.zeros(2, 4, dtype=torch.int32)), "page_table: shape"),
    (dict(cu=torch.zeros(2, dtype=torch.int32)), "cu_tokens: shape"),
    (dict(cu=torch.zeros(3, dtype=torch.int64)), "cu_tokens: dtype"),
])
def test_binding_checks_rows(over, msg):
    c, t = _tensors()
    t.update(over)
    with pytest.raises(B.LocksError, match=msg):
        C.rope_append_kv(c, t["k"], t["v"], t["kc"], t["vc"], t["pt"], t["sl"], cu_tokens=t.get("cu"))


def test_binding_reaches_the_device_check_and_checks_stores():
    c, t = _tensors()
    with pytest.raises(B.LocksError, match="device tensors"):
        C.rope_append_kv(c, t["k"], t["v"], t["kc"], t["vc"], t["pt"], t["sl"])
    store = C.alloc_q8_cache(c, device="cpu")
    assert store.k.dtype == torch.int8 and tuple(store.v_scale.shape) == (6, 2)
    with pytest.raises(B.LocksError, match="int8 or float8_e4m3fn"):
        C.alloc_q8_cache(c, torch.uint8, "cpu")
    q, ws = torch.zeros(2, 8, 128, dtype=torch.bfloat16), torch.zeros(64, dtype=torch.uint8)
    out, lse = torch.zeros(2, 8, 128), torch.zeros(2, 8)
    bad = C.Q8Cache(store.k, store.v.view(torch.float8_e4m3fn), store.k_scale, store.v_scale)
    with pytest.raises(B.LocksError, match="cache.v: dtype"):
        C.q8_dense_attend(c, q, bad, t["pt"], t["sl"], ws, out, lse)
    bad = C.Q8Cache(store.k, store.v, store.k_scale[:5], store.v_scale)
    with pytest.raises(B.LocksError, match="cache.k_scale: shape"):
        C.q8_dense_attend(c, q, bad, t["pt"], t["sl"], ws, out, lse)
    with pytest.raises(B.LocksError, match="page_ids: shape"):
        C.q8_sparse_attend(c, q, store, t["pt"], t["sl"], torch.zeros(2, 2, 3, dtype=torch.int32), ws, out, lse)
    with pytest.raises(B.LocksError, match="device tensors"):
        C.q8_dense_attend(c, q, store, t["pt"], t["sl"], ws, out, lse)


def test_rope_table_is_the_angles():
    t = C.rope_table(50, 64, device="cpu")
    assert t.shape == (50, 64) and t.dtype == torch.float32
    a = 49 * 10000.0 ** (-2.0 * 31 / 64)
    assert abs(float(t[49, 31]) - torch.tensor(a, dtype=torch.float64).cos().item()) < 1e-7
    assert float(t[0, :32].min()) == 1.0 and float(t[0, 32:].abs().max()) == 0.0
