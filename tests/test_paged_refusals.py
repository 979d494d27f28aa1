"""Host side of the paged-cache entry points (no GPU needed): every argument that breaks the rules of the header
is refused before anything is launched, and the kernels' own checks of lengths, row ranges and pages, compiled for
the host."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2504_08378_amd import binding as B
from paper_2504_08378_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
EINVAL, ENULL, ESHAPE, EWORKSPACE = -1, -2, -3, -4
CTX = C.create_string_buffer(4096)   # a context of zeros: no workspace, so a call that passes every check ends there
ONE = 4096                           # some 16-byte aligned address; no call reaches it


def _structs(cache=None, batch=None):
    c = dict(k_pages=ONE, v_pages=ONE, page_stride=2 * 16 * 64, n_pages=4, page_tokens=16, n_kv_heads=2, head_dim=64)
    b = dict(n_seqs=3, table_stride=5, n_rows=9, max_q_len=9, page_table=ONE, kv_len=ONE, q_start=ONE)
    c.update(cache or {})
    b.update(batch or {})
    return B.PagedCacheStruct(**c), B.PagedBatchStruct(**b)


def _append(cache=None, batch=None, **kw):
    a = dict(ctx=CTX, heads=4, theta=1e4, qg=None, kg=None, eps=1e-5, pos=None, qkv=ONE, ld=512, q=ONE, q_ld=256)
    a.update(kw)
    c, b = _structs(cache, batch)
    return B.lib().af_paged_append(a["ctx"], C.byref(c), C.byref(b), a["heads"], a["theta"], a["qg"], a["kg"], a["eps"],
                                   a["pos"], a["qkv"], a["ld"], a["q"], a["q_ld"])


def _attention(cache=None, batch=None, **kw):
    a = dict(ctx=CTX, heads=4, scale=0.0, window=0, sinks=0, q=ONE, q_ld=256, out=ONE, out_ld=256)
    a.update(kw)
    c, b = _structs(cache, batch)
    return B.lib().af_paged_attention(a["ctx"], C.byref(c), C.byref(b), a["heads"], a["scale"], a["window"], a["sinks"],
                                      a["q"], a["q_ld"], a["out"], a["out_ld"])


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(B.LIB_PATH):
        build.build(verbose=False)


CACHE = [({"k_pages": None}, ENULL), ({"v_pages": None}, ENULL), ({"k_pages": ONE + 8}, ESHAPE), ({"v_pages": ONE + 2}, ESHAPE),
         ({"n_pages": 0}, EINVAL), ({"n_pages": -1}, EINVAL), ({"n_kv_heads": 0}, EINVAL), ({"n_kv_heads": 3}, ESHAPE),
         ({"head_dim": 32}, ESHAPE), ({"head_dim": 96}, ESHAPE), ({"head_dim": 256}, ESHAPE), ({"page_tokens": 8}, ESHAPE),
         ({"page_tokens": 24}, ESHAPE), ({"page_tokens": 512}, ESHAPE), ({"page_tokens": 0}, ESHAPE), ({"page_tokens": -16}, ESHAPE),
         ({"page_stride": 2 * 16 * 64 - 8}, ESHAPE), ({"page_stride": 2 * 16 * 64 + 4}, ESHAPE), ({"page_stride": -4096}, ESHAPE)]
BATCH = [({"page_table": None}, ENULL), ({"kv_len": None}, ENULL), ({"n_seqs": 0}, EINVAL), ({"n_seqs": 1025}, EINVAL),
         ({"table_stride": 0}, EINVAL), ({"table_stride": (1 << 26) + 1}, EINVAL), ({"n_rows": -1}, EINVAL),
         ({"n_rows": (1 << 22) + 1}, EINVAL), ({"max_q_len": 0}, EINVAL), ({"q_start": None}, EINVAL),
         ({"q_start": None, "n_rows": 3}, EINVAL), ({"q_start": None, "n_rows": 4, "max_q_len": 1}, EINVAL)]


@pytest.mark.parametrize("call", [_append, _attention])
def test_cache_and_batch(call):
    for change, status in CACHE:
        assert call(cache=change) == status, change
    for change, status in BATCH:
        assert call(batch=change) == status, change
    assert call() == EWORKSPACE
    assert call(cache={"page_stride": 4096, "page_tokens": 32}) == EWORKSPACE
    assert call(batch={"q_start": None, "n_rows": 3, "max_q_len": 1}) == EWORKSPACE
    assert call(batch={"n_rows": 0}) == EWORKSPACE and call(batch={"n_rows": 0}, q=None) == EWORKSPACE
    assert call(heads=0) == EINVAL and call(heads=5) == ESHAPE and call(heads=-4) == EINVAL
    assert call(heads=1026) == EINVAL
    assert call(batch={"n_rows": 1 << 22}, heads=512) == EINVAL
    assert call(ctx=None) == ENULL
    assert B.lib().af_paged_append(CTX, None, None, 4, 1e4, None, None, 1e-5, None, ONE, 512, ONE, 256) == ENULL
    assert B.lib().af_paged_attention(CTX, None, None, 4, 0.0, 0, 0, ONE, 256, ONE, 256) == ENULL


def test_append_arguments():
    inf, nan = float("inf"), float("nan")
    for change, status in [({"qkv": None}, ENULL), ({"q": None, "q_ld": 0}, EWORKSPACE), ({"qkv": ONE + 8}, ESHAPE),
                           ({"q": ONE + 8}, ESHAPE), ({"ld": 504}, ESHAPE), ({"ld": 516}, ESHAPE), ({"q_ld": 248}, ESHAPE),
                           ({"q_ld": 260}, ESHAPE), ({"qg": ONE + 2}, ESHAPE), ({"kg": ONE + 8}, ESHAPE), ({"theta": 0.0}, EINVAL),
                           ({"theta": -1.0}, EINVAL), ({"theta": inf}, EINVAL), ({"theta": nan}, EINVAL), ({"eps": -1.0}, EINVAL),
                           ({"eps": nan}, EINVAL), ({"eps": inf}, EINVAL), ({"ld": 520, "q_ld": 512}, EWORKSPACE)]:
        assert _append(**change) == status, change


def test_attention_arguments():
    for change, status in [({"q": None}, ENULL), ({"out": None}, ENULL), ({"q": ONE + 2}, ESHAPE), ({"out": ONE + 8}, ESHAPE),
                           ({"q_ld": 248}, ESHAPE), ({"out_ld": 252}, ESHAPE), ({"q_ld": 257}, ESHAPE), ({"window": -1}, EINVAL),
                           ({"sinks": -1}, EINVAL), ({"scale": float("inf")}, EINVAL), ({"scale": float("nan")}, EINVAL),
                           ({"window": 7, "sinks": 9, "scale": -0.5}, EWORKSPACE)]:
        assert _attention(**change) == status, change


SOURCE = """
#include "paged.h"
extern "C" int seq(int table_stride, int shift, int ragged, int n_rows, int max_q, int row0, int row1, int len, int* out) {
  PagedView v{};
  static const int32_t some = 0;
  v.table_stride = table_stride; v.page_shift = shift; v.q_start = ragged ? &some : nullptr;
  v.n_rows = n_rows; v.max_q_len = max_q;
  PagedSeq s;
  const bool ok = paged_seq_check(v, row0, row1, len, &s);
  out[0] = s.row0; out[1] = s.q_len; out[2] = s.len;
  return ok;
}
extern "C" int page(int n_pages, int id) { PagedView v{}; v.n_pages = n_pages; return paged_page_ok(v, id); }
extern "C" long long offset(long long page_stride, int shift, int page, int h, int j, int hd) {
  PagedView v{}; v.page_stride = page_stride; v.page_shift = shift;
  return (long long)paged_offset(v, page, h, j, hd);
}
template <int TK> static int tiles_of(int p0, int p1, int window, int n_sink, int* starts, int most) {
  const PagedTiles t = paged_tiles<TK>(p0, p1, window, n_sink);
  for (int i = 0; i < t.n && i < most; ++i) starts[i] = paged_tile_start<TK>(t, i);
  return t.n;
}
extern "C" int tiles(int tk, int p0, int p1, int window, int n_sink, int* starts, int most) {
  return tk == 32 ? tiles_of<32>(p0, p1, window, n_sink, starts, most) : tiles_of<16>(p0, p1, window, n_sink, starts, most);
}
extern "C" int seen(int key, int place, int window, int n_sink) { return paged_seen(key, place, window, n_sink); }
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    d = tmp_path_factory.mktemp("paged")
    src, so = str(d / "paged.hip"), str(d / "paged.so")
    open(src, "w").write(SOURCE)
    subprocess.run([HIPCC, *build.HIPCC_FLAGS, "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "-shared", src,
                    "-o", so], check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    lib = C.CDLL(so)
    lib.offset.restype = C.c_longlong
    lib.offset.argtypes = [C.c_longlong] + [C.c_int] * 5
    return lib


def test_lengths_and_row_ranges(host):
    out = (C.c_int * 3)()
    big = 2 ** 31 - 1
    for ragged, row0, row1, length, ok in [
            (1, 0, 5, 5, 1), (1, 3, 3, 0, 1), (1, 0, 9, 80, 1), (1, 0, 5, 4, 0), (1, 5, 4, 9, 0), (1, -1, 2, 9, 0), (1, 4, 11, 9, 0),
            (1, 0, 10, 20, 0), (1, 0, 2, -1, 0), (1, 0, 2, 81, 0), (1, 0, 2, big, 0), (1, -2 ** 31, big, big, 0), (1, big, -2 ** 31, 5, 0),
            (0, 2, 3, 0, 1), (0, 2, 3, 80, 1), (0, 2, 3, 81, 0), (0, 2, 3, -1, 0)]:
        assert host.seq(5, 4, ragged, 10, 9, row0, row1, length, out) == ok, (ragged, row0, row1, length)
        if ok:
            assert list(out) == [row0, row1 - row0, length]
        else:
            assert list(out)[1:] == [0, 0]


def test_pages_and_offsets(host):
    for n, page, ok in [(4, 0, 1), (4, 3, 1), (4, 4, 0), (4, -1, 0), (1, 2 ** 31 - 1, 0), (2 ** 31 - 1, -2 ** 31, 0)]:
        assert host.page(n, page) == ok
    for shift, kv, hd in ((4, 2, 64), (8, 64, 128)):
        stride = (kv << shift) * hd + 8
        for page, h, j in ((0, 0, 0), (7, kv - 1, 12345), (100000, 1, (1 << 30) - 1)):
            want = page * stride + ((h << shift) + j % (1 << shift)) * hd
            assert host.offset(stride, shift, page, h, j, hd) == want   # past 32 bits in a long cache


@pytest.mark.parametrize("tk", [16, 32])
def test_tiles_hold_every_key_that_is_seen_once(host, tk):
    starts = (C.c_int * 4096)()
    for p0, p1 in ((0, 0), (5, 5), (63, 64), (127, 127), (128, 128), (0, 300), (777, 777), (500, 900), (1000, 1015)):
        for window in (0, 1, 2, 15, 16, 17, 64, 100, 128, 129, 500, 2 ** 31 - 1):
            for sinks in (0, 1, 16, 64, 100, 129, 600, 2 ** 31 - 1):
                n = host.tiles(tk, p0, p1, window, sinks, starts, 4096)
                held = [k for i in range(n) for k in range(starts[i], starts[i] + tk)]
                assert len(held) == len(set(held)) and all(starts[i] % 16 == 0 for i in range(n))
                see = {j for p in (p0, p1) for j in range(p1 + 1) if host.seen(j, p, window, sinks)}
                assert see <= set(held) and held[-1] >= p1 and starts[n - 1] <= p1
                assert see == {j for p in (p0, p1) for j in range(p + 1) if not window or j > p - window or j < sinks}
                wide = p1 + 1 if not window else min(p1 + 1, p1 - max(0, p0 - window + 1) + 1 + min(sinks, max(0, p0 - window + 1)))
                # no tile that nothing needs, but where the first tokens and the window end inside one, its start is moved to
                # sixteen keys and less than a tile lies between the two
                assert n <= wide // tk + 4
    assert host.tiles(tk, -1, -1, 0, 0, starts, 4096) == 0
    far = 2 ** 30 - 1
    assert host.tiles(tk, far, far, 2 ** 31 - 1, 2 ** 31 - 1, starts, 4096) == 2 ** 30 // tk
    assert host.tiles(tk, far, far, 100, 2 ** 31 - 1, starts, 4096) == 2 ** 30 // tk
    assert host.tiles(tk, far, far, 100, 4, starts, 4096) == 1 + (112 + tk - 1) // tk  # seen from far - 99 = 12 mod 16 on
