"""Refusals of the calls on a paged 8-bit cache: found on the host, before anything is launched (no GPU is needed)."""
import ctypes as C
import os

import pytest
import torch


@pytest.fixture(scope="module")
def amd():
    import paper_2408_11850_amd as amd
    if not os.path.exists(amd.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    amd.load_library()
    return amd


# addresses far from each other that are never read
MB = 1 << 20
K, V, SCALE, TABLE, LEN, Q, OUT, LSE, WORK, ROWS, W, POS, NEWK, NEWV, KEPT, W2 = (i * 64 * MB for i in range(1, 17))
CACHE = dict(k=K, v=V, scale=SCALE, table=TABLE, len=LEN, n_pages=20, n_kv_heads=2, head_dim=128, n_seqs=3, max_pages=4, table_ld=5)
LONG = dict(max_pages=500, table_ld=500)           # what needs a workspace
BAD_CACHES = [dict(k=None), dict(v=None), dict(scale=None), dict(table=None), dict(len=None), dict(n_pages=0), dict(n_pages=-1), dict(n_kv_heads=0),
              dict(n_kv_heads=5000), dict(head_dim=96), dict(head_dim=0), dict(head_dim=256), dict(n_seqs=0), dict(n_seqs=65536),
              dict(n_seqs=60000, n_kv_heads=20), dict(max_pages=0), dict(max_pages=(1 << 20) + 1, table_ld=1 << 21), dict(table_ld=3), dict(max_pages=1 << 20, table_ld=1 << 20, n_kv_heads=32),
              dict(k=K + 8), dict(v=V + 1), dict(scale=SCALE + 4), dict(table=TABLE + 2), dict(len=LEN + 1)]


def _cache(amd, **change):
    d = {**CACHE, **change}
    return amd.QuantCacheDesc(*(d[n] for n, _ in amd.QuantCacheDesc._fields_))


def _split(change):
    return {k: v for k, v in change.items() if k in CACHE}, {k: v for k, v in change.items() if k not in CACHE}


def _attend(amd, **change):
    c, o = _split(change)
    a = {**dict(q=Q, ldq=1024, rows=ROWS, n=7, heads=8, by=0.1, window=0, sinks=0, out=OUT, lse=LSE, work=WORK, none=False), **o}
    cache = _cache(amd, **c)
    return amd.load_library().spec_attend_quant(None if a["none"] else C.byref(cache), a["q"], a["ldq"], a["rows"], a["n"], a["heads"], a["by"],
                                                a["window"], a["sinks"], a["out"], a["lse"], a["work"], None)


ROW_CHANGES = [dict(none=True), dict(q=None), dict(ldq=1000), dict(ldq=1028), dict(ldq=-1024), dict(q=Q + 8), dict(n=0), dict(n=-3),
               dict(n=(1 << 23) + 1), dict(heads=0), dict(heads=7), dict(heads=8192, ldq=1 << 20), dict(rows=None), dict(rows=ROWS + 2), dict(by=0.0),
               dict(by=-1.0), dict(by=float("nan")), dict(by=float("inf")), dict(window=-1), dict(sinks=-1)]


@pytest.mark.parametrize("change", BAD_CACHES + ROW_CHANGES + [
    dict(out=None), dict(out=OUT + 8), dict(lse=LSE + 2), dict(work=WORK + 8), dict(work=None, **LONG), dict(out=Q), dict(out=Q + 1024 * 2 * 6 + 2032), dict(lse=OUT + 16),
    dict(work=OUT, **LONG), dict(work=LSE, **LONG), dict(out=K + 16), dict(lse=SCALE), dict(work=V, **LONG), dict(out=TABLE), dict(lse=LEN), dict(lse=ROWS), dict(work=Q + 16, **LONG)], ids=str)
def test_attend_refuses(amd, change):
    assert _attend(amd, **change) == amd.SPEC_E_INVAL


@pytest.mark.parametrize("change", BAD_CACHES + ROW_CHANGES + [
    dict(lse=None), dict(weight=None), dict(weight=W + 2), dict(lse=LSE + 1), dict(ldw=255), dict(ldw=1 << 41), dict(weight=Q), dict(weight=LSE),
    dict(weight=SCALE), dict(weight=ROWS), dict(weight=K + 64), dict(work=None, n=4000), dict(work=W + 16, n=4000), dict(work=LSE, n=4000), dict(work=WORK + 4)],
    ids=str)
def test_weigh_refuses(amd, change):
    c, o = _split(change)
    a = {**dict(q=Q, ldq=1024, lse=LSE, rows=ROWS, n=7, heads=8, by=0.1, window=0, sinks=0, weight=W, ldw=256, work=WORK, none=False), **o}
    cache = _cache(amd, **c)
    assert amd.load_library().spec_weigh_quant(None if a["none"] else C.byref(cache), a["q"], a["ldq"], a["lse"], a["rows"], a["n"], a["heads"],
                                               a["by"], a["window"], a["sinks"], a["weight"], a["ldw"], a["work"], None) == amd.SPEC_E_INVAL


@pytest.mark.parametrize("change", BAD_CACHES + [
    dict(none=True), dict(k2=None), dict(v2=None), dict(type=2), dict(n=0), dict(rows=None), dict(heads=7), dict(heads=0), dict(ldk=255), dict(ldv=100), dict(ldq=1000),
    dict(ldk=-256), dict(k2=NEWK + 1), dict(type=0, v2=NEWV + 2), dict(q=Q + 1), dict(qo=OUT + 8), dict(pos=POS + 2), dict(qo=None), dict(q=None),
    dict(theta=0.5), dict(theta=-1.0), dict(theta=float("nan")), dict(theta=float("inf")), dict(qo=NEWK), dict(qo=NEWV + 512), dict(qo=Q + 16),
    dict(qo=Q, ldq=1032), dict(qo=Q, type=0, ldq=1024), dict(qo=K), dict(qo=POS), dict(qo=ROWS), dict(k2=K), dict(v2=SCALE), dict(q=V + 16)], ids=str)
def test_append_refuses(amd, change):
    c, o = _split(change)
    a = {**dict(k2=NEWK, ldk=256, v2=NEWV, ldv=256, type=1, rows=ROWS, n=7, q=Q, ldq=1024, heads=8, theta=1e4, pos=POS, qo=OUT, none=False), **o}
    cache = _cache(amd, **c)
    assert amd.load_library().spec_append_quant(None if a["none"] else C.byref(cache), a["k2"], a["ldk"], a["v2"], a["ldv"], a["type"], a["rows"], a["n"],
                                                a["q"], a["ldq"], a["heads"], a["theta"], a["pos"], a["qo"], None) == amd.SPEC_E_INVAL


TO = dict(k=K + 32 * MB, v=V + 32 * MB, scale=SCALE + 32 * MB, table=TABLE + 32 * MB, len=LEN + 32 * MB, n_pages=20, n_kv_heads=2, head_dim=128, n_seqs=3,
          max_pages=2, table_ld=2)


@pytest.mark.parametrize("change", BAD_CACHES + [dict(to=t) for t in BAD_CACHES if "max_pages" not in t and "table_ld" not in t] + [
    dict(none=True), dict(to=dict(n_kv_heads=3)), dict(to=dict(head_dim=64)), dict(to=dict(n_seqs=2)), dict(weight=None), dict(kept=None), dict(w2=None),
    dict(weight=W + 2), dict(kept=KEPT + 1), dict(w2=W2 + 2), dict(ldw=255), dict(ldt=99), dict(budget=0), dict(budget=-1), dict(budget=129), dict(sinks=-1),
    dict(recent=-1), dict(sinks=60, recent=41), dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1), dict(kept=W), dict(w2=W + 4), dict(w2=KEPT), dict(kept=K), dict(w2=TABLE),
    dict(to=dict(len=LEN)), dict(to=dict(len=TABLE)), dict(to=dict(k=K + 16)), dict(to=dict(k=V)), dict(to=dict(scale=W)), dict(to=dict(len=KEPT)),
    dict(to=dict(table=KEPT)), dict(to=dict(len=TABLE + 32 * MB))], ids=str)
def test_evict_refuses(amd, change):
    c, o = _split(change)
    a = {**dict(weight=W, ldw=256, to={}, budget=100, sinks=4, recent=20, kept=KEPT, w2=W2, ldt=100, none=False), **o}
    cache, to = _cache(amd, **c), _cache(amd, **{**TO, **a["to"]})
    assert amd.load_library().spec_evict_quant(None if a["none"] else C.byref(cache), a["weight"], a["ldw"], C.byref(to), a["budget"], a["sinks"], a["recent"],
                                               a["kept"], a["w2"], a["ldt"], None) == amd.SPEC_E_INVAL


def test_workspaces(amd):
    """0 for what is refused and for rows whose attention is one launch; else the parts of all rows, whatever the row starts hold."""
    lib = amd.load_library()
    size = lambda n, window=0, sinks=0, rows=ROWS, f=lib.spec_attend_quant_workspace_bytes, **c: f(C.byref(_cache(amd, **c)), rows, n, 8, window, sinks)
    need = size(3, **LONG)
    assert need > 0 and need % (3 * 8 * 130 * 4) == 0 and need // (3 * 8 * 130 * 4) <= 64
    assert 0 < size(3, window=300, **LONG) < need and size(3, window=500 * 64, **LONG) == need
    weigh = lib.spec_weigh_quant_workspace_bytes
    assert size(3, f=weigh, **LONG) == 0 and size(4000, f=weigh) % (3 * 2 * 4 * 64 * 4) == 0 < size(4000, f=weigh)


def test_python_calls_refuse(amd):
    h = torch.zeros(2, 2, 64, 128, dtype=torch.float8_e4m3fn)
    with pytest.raises(ValueError):
        amd.Fp8Cache(h, h, torch.zeros(2, 2, 2), torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
