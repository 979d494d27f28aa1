"""GPU parity of the paged-cache operators against a plain implementation in 64 bits, written here row by row:
af_paged_append (norms, rotation, rows to their pages) and af_paged_attention (single tokens, a few, prompts;
window and first tokens; what no row sees; batches as they occur).

Tolerances.  A result is fp32 arithmetic rounded to fp16 once: half a unit in the last place (2^-11 of the
value; 2^-25 below the normal range) plus the fp32 error, of the size of the sums' terms: 2^-17 of sum |terms| covers
some 64 roundings.  Attention of prompts holds its weights in fp16 for the matrix cores: each is off by 2^-11 of itself at
most, which adds 2^-11 sum w|v| / sum w."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2504_08378_amd import binding as B
from gpu_util import ctx, to_dev, to_host  # noqa: F401

pytestmark = pytest.mark.gpu


class Batch:
    """A paged cache and a ragged batch, on the host and on the device.  lens: (cached tokens with the new ones, new)."""

    def __init__(self, lens, kv_heads, hd, page, seed=0, single=False, spare_rows=0, spare_table=2, stale=np.nan, gap=0,
                 max_q_len=None):
        rng = np.random.default_rng(seed)
        self.lens, self.kv, self.hd, self.page = lens, kv_heads, hd, page
        need = [-(-n // page) for n, _ in lens]
        self.n_pages = sum(need) + 3
        order = rng.permutation(self.n_pages)
        width = max(need + [1]) + spare_table
        self.table = np.full((len(lens), width), -7, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at: at + n]
            at += n
        shape = (self.n_pages, kv_heads, page, hd)
        self.K, self.V = (np.full(shape, stale, np.float16) for _ in range(2))
        for b, (n, _) in enumerate(lens):
            for j in range(n):
                pg = self.table[b, j // page]
                self.K[pg, :, j % page], self.V[pg, :, j % page] = rng.standard_normal((2, kv_heads, hd))
        self.start = np.concatenate([[0], np.cumsum([q for _, q in lens])]).astype(np.int32)
        self.rows = (len(lens) if single else int(self.start[-1])) + spare_rows
        self.single = single
        self.gap = gap
        self.max_q = max_q_len if max_q_len is not None else max([q for _, q in lens] + [1])
        self.rng = rng

    def upload(self):
        def pages(a):
            if not self.gap:
                return to_dev(a)
            big = torch.full((self.n_pages, a[0].size + self.gap), float("nan"), dtype=torch.float16, device="cuda")
            v = big[:, : a[0].size].view(self.n_pages, *a.shape[1:])
            v.copy_(to_dev(a))
            return v
        self.Kd, self.Vd = pages(self.K), pages(self.V)
        self.cache = B.PagedCache(self.Kd, self.Vd)
        kv_len = to_dev(np.array([n for n, _ in self.lens], np.int32))
        if self.single:
            self.batch = B.PagedBatch(to_dev(self.table), kv_len)
        else:
            self.batch = B.PagedBatch(to_dev(self.table), kv_len, to_dev(self.start), self.rows, self.max_q)
        return self

    def tokens(self):
        """(row, sequence, place) of every new token."""
        for b, (n, q) in enumerate(self.lens):
            for i in range(q):
                yield (b if self.single else int(self.start[b])) + i, b, n - q + i

    def keys(self, b, places):
        pg, slot = self.table[b, places // self.page], places % self.page
        return self.K[pg, :, slot].astype(np.float64), self.V[pg, :, slot].astype(np.float64)


def seen(place, window, sinks):
    j = np.arange(place + 1)
    return j if not window else j[(j > place - window) | (j < sinks)]


def attend(bt, q, heads, window=0, sinks=0, scale=None, bad=()):
    """{row: (result [heads][hd], sum w|v| / sum w)} in 64 bits.  bad: (sequence, table entry) without a page."""
    rep, out = heads // bt.kv, {}
    scale = 1 / np.sqrt(bt.hd) if scale is None else scale
    for row, b, place in bt.tokens():
        j = seen(place, window, sinks)
        j = j[[(b, x // bt.page) not in bad for x in j]] if bad else j
        o, mag = np.zeros((2, heads, bt.hd))
        if len(j):
            K, V = bt.keys(b, j)
            x = q[row].astype(np.float64).reshape(bt.kv, rep, bt.hd)
            with np.errstate(invalid="ignore", over="ignore"):
                s = np.einsum("grd,jgd->grj", x, K) * scale
                w = np.exp(s - s.max(-1, keepdims=True))
                w /= w.sum(-1, keepdims=True)
                o = np.einsum("grj,jgd->grd", w, V).reshape(heads, bt.hd)
                mag = np.einsum("grj,jgd->grd", w, np.abs(V)).reshape(heads, bt.hd)
        out[row] = o, mag
    return out


def check(got, ref, heads, hd, weights16=False, untouched=None):
    for row in range(got.shape[0]):
        g = got[row].astype(np.float64).reshape(heads, hd)
        if row not in ref:
            assert np.all(g == untouched), row
            continue
        o, mag = ref[row]
        fine = np.isfinite(o)
        assert np.array_equal(np.isnan(o), np.isnan(g)) and np.array_equal(o[~fine & ~np.isnan(o)], g[~fine & ~np.isnan(o)]), row
        tol = 2.0 ** -11 * np.abs(o) + 2.0 ** -25 + 2.0 ** -17 * mag + (2.0 ** -11 * mag if weights16 else 0)
        worst = np.max(np.abs(g - o)[fine] - tol[fine], initial=-1.0)
        assert worst <= 0, (row, worst)


def run(ctx, bt, heads, q=None, fill=5.0, err=0, pad=0, **kw):
    bt.upload()
    if q is None:
        q = (2 * bt.rng.standard_normal((bt.rows, heads * bt.hd))).astype(np.float16)
    qd = to_dev(np.concatenate([q, np.full((bt.rows, pad), np.nan, np.float16)], 1))[:, : heads * bt.hd]
    out = torch.full((bt.rows, heads * bt.hd + pad), fill, dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    ctx.paged_attention(bt.cache, bt.batch, qd, out[:, : heads * bt.hd], heads, **kw)
    ctx.synchronize()
    assert ctx.last_device_error() == err
    got = to_host(out)
    assert np.all(got[:, heads * bt.hd:] == fill)
    return q, got[:, : heads * bt.hd]


HEADS = [(1, 1, 64), (4, 4, 128), (8, 1, 128), (6, 2, 64), (9, 3, 64), (20, 1, 64), (64, 8, 128)]


@pytest.mark.parametrize("heads,kv,hd", HEADS)
@pytest.mark.parametrize("page", [16, 64, 256])
def test_single_tokens(ctx, heads, kv, hd, page):
    """One token per sequence, lengths from none over one to several steps, on both sides of every step and page."""
    lens = [(n, 1 if n else 0) for n in (1, 0, 2, 15, 16, 17, 31, 33, 64, 127, 128, 129, 255, 257, 640)]
    bt = Batch(lens, kv, hd, page, seed=heads + page, single=True)
    q, got = run(ctx, bt, heads)
    assert np.all(got[1] == 0)  # nothing cached, nothing seen
    ref = attend(bt, q, heads)
    ref[1] = np.zeros((heads, hd)), np.zeros((heads, hd))
    check(got, ref, heads, hd)


@pytest.mark.parametrize("heads,kv,hd", [(8, 8, 128), (16, 2, 128), (8, 2, 64)])
@pytest.mark.parametrize("n", [3000, 9001])
def test_one_long_sequence(ctx, heads, kv, hd, n):
    bt = Batch([(n, 1)], kv, hd, 32, seed=n, single=True)
    for _ in range(2):  # the second call finds the counters the first one left
        q, got = run(ctx, bt, heads)
        check(got, attend(bt, q, heads), heads, hd)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (16, 16), (100, 4), (128, 0), (128, 130), (1000, 40), (2 ** 31 - 1, 9)])
@pytest.mark.parametrize("single", [True, False])
def test_window_and_first_tokens(ctx, window, sinks, single):
    heads, kv, hd = 6, 2, 64
    lens = [(n, 1) for n in (1, 4, 17, 100, 129, 300, 777)] if single else [(70, 70), (333, 200), (500, 3), (130, 129), (40, 17)]
    bt = Batch(lens, kv, hd, 16, seed=window % 1000 + sinks, single=single)
    q, got = run(ctx, bt, heads, window=window, n_sink=sinks)
    check(got, attend(bt, q, heads, window, sinks), heads, hd, weights16=not single)


@pytest.mark.parametrize("heads,kv,hd", [(1, 1, 128), (4, 4, 64), (8, 1, 128), (6, 2, 64), (20, 1, 64), (32, 8, 128)])
@pytest.mark.parametrize("page", [16, 128])
def test_ragged_prompts(ctx, heads, kv, hd, page):
    """Prompts from one token to hundreds, with and without a past, an empty range among them, rows behind the last."""
    lens = [(1, 1), (40, 40), (300, 1), (64, 0), (0, 0), (129, 129), (260, 7), (257, 100), (65, 65), (18, 2), (331, 300)]
    bt = Batch(lens, kv, hd, page, seed=heads + hd, spare_rows=5)
    q, got = run(ctx, bt, heads)
    check(got, attend(bt, q, heads), heads, hd, weights16=True, untouched=5.0)


@pytest.mark.parametrize("new", [2, 3, 4, 5, 8, 9, 16, 17, 31, 33])
def test_a_few_new_tokens(ctx, new):
    """Drafted tokens behind a long past."""
    for heads, kv, hd in ((4, 4, 64), (8, 2, 128), (32, 2, 64)):
        bt = Batch([(new, new), (700 + new, new), (131, new)], kv, hd, 16, seed=new)
        q, got = run(ctx, bt, heads)
        check(got, attend(bt, q, heads), heads, hd, weights16=True)


@pytest.mark.parametrize("heads,kv,hd", [(4, 4, 64), (8, 2, 128), (32, 8, 128), (16, 1, 64)])
@pytest.mark.parametrize("lens", [[(3000, 40)], [(5000, 17), (700, 130)], [(2600, 300), (1, 1), (900, 3), (40, 40)]])
def test_few_rows_of_many_keys(ctx, heads, kv, hd, lens):
    """Few workgroups, many keys: the rows' keys are shared out in pieces and joined; twice, for the counters; under a window that
    leaves pieces in which rows see nothing; and with values that are not finite, which are seen by some rows only."""
    for window, sinks in ((0, 0), (0, 0), (1500, 70)):
        bt = Batch(lens, kv, hd, 16, seed=heads + window, stale=np.nan)
        n, new = lens[0]
        bt.V[bt.table[0, (n - 5) // 16], 0, (n - 5) % 16, 3] = np.inf
        q, got = run(ctx, bt, heads, window=window, n_sink=sinks)
        check(got, attend(bt, q, heads, window, sinks), heads, hd, weights16=True)


@pytest.mark.parametrize("lens", [[2900] * 16, [100 + 250 * i for i in range(16)], [700 - 5 * i for i in range(70)]])
@pytest.mark.parametrize("new", [1, 2])
def test_many_keys_of_many_sequences(ctx, lens, new):
    """Several units of keys for every workgroup: as many for each sequence, as fits; for sequences that differ; for more than 64."""
    heads, kv, hd = 16, 8, 64
    for window, sinks in ((0, 0), (1500, 20)):
        bt = Batch([(n, new) for n in lens], kv, hd, 64, seed=len(lens), single=new == 1)
        q, got = run(ctx, bt, heads, window=window, n_sink=sinks)
        check(got, attend(bt, q, heads, window=window, sinks=sinks), heads, hd)


def test_smallest_workspace(ctx):
    """A workspace for one small token: fewer stretches and pieces, the same results."""
    heads, kv, hd = 16, 1, 128
    small = B.Context(0, max_in=64, max_out=64, max_batch=1)
    try:
        for lens, single in (([(9000, 1), (300, 1)], True), ([(4000, 40), (900, 1)], False)):
            bt = Batch(lens, kv, hd, 16, seed=5, single=single)
            q, got = run(small, bt, heads)
            check(got, attend(bt, q, heads), heads, hd, weights16=not single)
    finally:
        small.close()


@pytest.mark.parametrize("single", [True, False])
def test_as_many_sequences_as_there_may_be(ctx, single):
    heads, kv, hd = 2, 1, 64
    rng = np.random.default_rng(3)
    lens = [(int(n), 1 if single else int(min(n, q))) for n, q in zip(rng.integers(1, 40, 1024), rng.choice([0, 1, 2, 12], 1024))]
    lens[700] = (2500, 1 if single else 300)
    bt = Batch(lens, kv, hd, 16, seed=3, single=single)
    q, got = run(ctx, bt, heads)
    check(got, attend(bt, q, heads), heads, hd, weights16=not single)
    run_append(ctx, bt, heads)


@pytest.mark.parametrize("single", [True, False])
def test_strides_scale_and_spaced_pages(ctx, single):
    heads, kv, hd = 6, 3, 64
    lens = [(200, 1), (33, 1)] if single else [(90, 80), (20, 20), (400, 2)]
    bt = Batch(lens, kv, hd, 32, seed=4, single=single, gap=64, spare_table=5)
    for scale in (0.25, -0.1):
        q, got = run(ctx, bt, heads, pad=24, scale=scale)
        check(got, attend(bt, q, heads, scale=scale), heads, hd, weights16=not single)


@pytest.mark.parametrize("new", [1, 2, 70])
def test_offsets_beyond_32_bits(ctx, new):
    """Pages and rows that lie 2^32 elements and more apart: the same bits as with near ones."""
    heads, kv, hd = 4, 2, 64
    far, near = (Batch([(90, new)] * 2, kv, hd, 16, seed=8, gap=gap, single=new == 1).upload() for gap in (2 ** 30, 0))
    assert int(far.table.max()) * 2 ** 30 > 2 ** 32
    width = heads * hd
    x = torch.randn((far.rows, (heads + 2 * kv) * hd), device="cuda").half()
    results = []
    for bt in (far, near):
        def rows_of(w):
            apart = 2 ** 32 // (bt.rows - 1) // 8 * 8 + 8 if new < 70 and bt is far else w
            return torch.empty((bt.rows - 1) * apart + w, dtype=torch.float16, device="cuda").as_strided((bt.rows, w), (apart, 1))
        qkv, q, out = rows_of(x.shape[1]), rows_of(width), rows_of(width)
        qkv.copy_(x)
        q.fill_(5.0)
        out.fill_(5.0)
        torch.cuda.synchronize()
        ctx.paged_append(bt.cache, bt.batch, qkv, q, heads)
        ctx.paged_attention(bt.cache, bt.batch, q, out, heads)
        ctx.synchronize()
        assert ctx.last_device_error() == 0
        results.append([to_host(t.contiguous()).view(np.uint16) for t in (q, out, bt.Kd, bt.Vd)])
        del qkv, q, out
    for a, b in zip(*results):
        assert np.array_equal(a, b)
    assert not np.any(results[0][1] == np.float16(5.0).view(np.uint16))
    del far, near, bt
    torch.cuda.empty_cache()


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("single", [True, False])
def test_what_a_row_does_not_see_does_not_enter(ctx, value, single):
    """Keys and values outside of the window, of later tokens of the same prompt and in unused slots hold `value`."""
    heads, kv, hd, window, sinks = 4, 2, 64, 20, 2
    lens = [(100, 1), (57, 1), (300, 1)] if single else [(100, 60), (57, 57), (300, 3)]
    bt = Batch(lens, kv, hd, 16, seed=9, single=single, stale=value)
    bt.K[bt.table[0, 0], :, 5], bt.V[bt.table[0, 0], :, 5] = value, value   # behind every window's start
    if not single:  # one token of the prompt: later rows see it, earlier ones do not
        bt.K[bt.table[1, 1], :, 9], bt.V[bt.table[1, 1], 0, 9, 3] = 1.0, value
        bt.V[bt.table[2, 299 // 16], :, 299 % 16] = value
    q, got = run(ctx, bt, heads, window=window, n_sink=sinks)
    ref = attend(bt, q, heads, window, sinks)
    check(got, ref, heads, hd, weights16=not single)
    assert any(np.all(np.isfinite(o)) for o, _ in ref.values())


@pytest.mark.parametrize("single", [True, False])
def test_special_values_that_are_seen(ctx, single):
    """An infinite value reaches its own dimension; a key of -inf scores has no weight; NaN reaches its key head's rows."""
    heads, kv, hd = 4, 2, 64
    bt = Batch([(150, 1), (40, 1)] if single else [(150, 90), (40, 40)], kv, hd, 16, seed=3, single=single)
    bt.V[bt.table[0, 2], 0, 3, 7] = np.inf
    bt.V[bt.table[1, 0], 1, 2, 1] = np.nan
    bt.K[bt.table[0, 1], 1, 4, 0] = np.inf
    q = (2 * bt.rng.standard_normal((bt.rows, heads * hd))).astype(np.float16)
    q[:, 2 * hd] = -np.abs(q[:, 2 * hd]) - 1   # both query heads of key head 1 score that key -inf
    q[:, 3 * hd] = -np.abs(q[:, 3 * hd]) - 1
    _, got = run(ctx, bt, heads, q=q)
    check(got, attend(bt, q, heads), heads, hd, weights16=not single)


@pytest.mark.parametrize("single", [True, False])
def test_wide_scores(ctx, single):
    """Scores far apart: one key takes everything; and all equal."""
    heads, kv, hd = 2, 1, 128
    bt = Batch([(500, 1)] if single else [(500, 300)], kv, hd, 64, seed=8, single=single)
    q = (30 * bt.rng.standard_normal((bt.rows, heads * hd))).astype(np.float16)
    q[0] = 0
    _, got = run(ctx, bt, heads, q=q)
    # scores of several hundred: their own fp32 error, some 2^-22 of them, multiplies the weights
    ref = {r: (o, mag * 8) for r, (o, mag) in attend(bt, q, heads).items()}
    check(got, ref, heads, hd, weights16=not single)


@pytest.mark.parametrize("single", [True, False])
def test_shared_pages(ctx, single):
    """Two sequences with the same first pages (and one of them twice in one table)."""
    heads, kv, hd = 4, 2, 64
    bt = Batch([(100, 1), (90, 1)] if single else [(100, 20), (90, 60)], kv, hd, 16, seed=2, single=single)
    bt.table[1, :3] = bt.table[0, :3]
    bt.table[0, 4] = bt.table[0, 1]
    q, got = run(ctx, bt, heads)
    check(got, attend(bt, q, heads), heads, hd, weights16=not single)


@pytest.mark.parametrize("bad_id", [-1, -2 ** 31, 10 ** 6, 2 ** 31 - 1])
@pytest.mark.parametrize("single", [True, False])
def test_a_page_that_does_not_exist_is_reported_and_not_seen(ctx, bad_id, single):
    heads, kv, hd = 4, 2, 64
    bt = Batch([(100, 1), (16, 1), (300, 1)] if single else [(100, 40), (16, 16), (300, 2)], kv, hd, 16, seed=6, single=single)
    bad = {(0, 2), (1, 0), (2, 11)}
    for b, e in bad:
        bt.table[b, e] = bad_id
    q, got = run(ctx, bt, heads, err=B.AF_DEVERR_PAGED)
    check(got, attend(bt, q, heads, bad=bad), heads, hd, weights16=not single)


def test_ranges_that_cannot_be_right_are_reported_and_left_alone(ctx):
    heads, kv, hd = 4, 2, 64
    for edit in ("negative length", "length beyond the table", "rows backwards", "rows beyond", "more rows than tokens", "more rows than said"):
        bt = Batch([(50, 20), (60, 30), (20, 10)], kv, hd, 16, seed=1, spare_rows=4, spare_table=0)
        lens = list(bt.lens)
        left = {1}
        if edit == "negative length":
            bt.lens = [lens[0], (-5, 30), lens[2]]
        elif edit == "length beyond the table":
            bt.lens = [lens[0], (65, 30), lens[2]]
        elif edit == "more rows than tokens":
            bt.lens = [lens[0], (29, 30), lens[2]]
        elif edit == "more rows than said":
            bt.max_q = 29
        elif edit == "rows backwards":
            bt.start[2] = 10
            left = {1, 2}
        else:
            bt.start[3] = bt.rows + 1
            left = {2}
        q, got = run(ctx, bt, heads, err=B.AF_DEVERR_PAGED)
        bt.lens = [l if b not in left else (l[0], 0) for b, l in enumerate(lens)]
        if edit == "rows backwards":  # the third range starts early: its rows are too many for its tokens
            bt.lens[2] = (lens[2][0], 0)
        check(got, attend(bt, q, heads), heads, hd, weights16=True, untouched=5.0)
    one = Batch([(50, 1), (-1, 1), (20, 1)], kv, hd, 16, single=True)
    one.table[1] = one.table[0]
    q, got = run(ctx, one, heads, err=B.AF_DEVERR_PAGED)
    one.lens[1] = (0, 0)
    check(got, attend(one, q, heads), heads, hd, untouched=5.0)


# ---- append ---------------------------------------------------------------------------------------------
def append_ref(bt, qkv, heads, theta=10000.0, gains=(None, None), eps=1e-5, pos=None):
    """{row: rotated [heads + kv][hd]} in 64 bits, with the magnitude of what enters each element."""
    hd, out = bt.hd, {}
    for row, b, place in bt.tokens():
        x = qkv[row].astype(np.float64).reshape(-1, hd)[: heads + bt.kv]
        for gain, at in ((gains[0], slice(0, heads)), (gains[1], slice(heads, None))):
            if gain is not None:
                x[at] = x[at] / np.sqrt((x[at] ** 2).mean(-1, keepdims=True) + eps) * gain.astype(np.float64)
        ang = (place if pos is None else int(pos[row])) * theta ** (-2.0 * np.arange(hd // 2) / hd)
        a, c = x[:, : hd // 2], x[:, hd // 2:]
        cs, sn = np.cos(ang), np.sin(ang)
        out[row] = np.concatenate([a * cs - c * sn, c * cs + a * sn], 1), np.tile(np.hypot(a, c), 2)
    return out


def run_append(ctx, bt, heads, in_place=False, no_q=False, pad=0, theta=10000.0, gains=(None, None), eps=1e-5, pos=None, err=0):
    bt.upload()
    width = (heads + 2 * bt.kv) * bt.hd
    qkv = bt.rng.standard_normal((bt.rows, width)).astype(np.float16)
    src = to_dev(np.concatenate([qkv, np.zeros((bt.rows, pad), np.float16)], 1))[:, :width]
    q_out = None if no_q else src[:, : heads * bt.hd] if in_place else \
        torch.full((bt.rows, heads * bt.hd), 5.0, dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    g = [None if v is None else to_dev(v) for v in gains]
    ctx.paged_append(bt.cache, bt.batch, src, q_out, heads, rope_theta=theta, q_gain=g[0], k_gain=g[1], eps=eps,
                     pos=None if pos is None else to_dev(pos))
    ctx.synchronize()
    assert ctx.last_device_error() == err
    K, V = bt.K.copy(), bt.V.copy()
    where = {r: (b, p) for r, b, p in bt.tokens()}
    Kg, qg = to_host(bt.Kd), None if no_q else to_host(q_out)
    for row, (x, mag) in append_ref(bt, qkv, heads, theta, gains, eps, pos).items():
        b, place = where[row]
        at = bt.table[b, place // bt.page], slice(None), place % bt.page
        # one rounding, and fp32 on the way: angle (2^-25 of a turn), norm, products
        tol = 2.0 ** -11 * np.abs(x) + 2.0 ** -25 + 2.0 ** -20 * mag
        assert np.all(np.abs(Kg[at].astype(np.float64) - x[heads:]) <= tol[heads:]), row
        K[at] = Kg[at]
        V[at] = qkv[row].reshape(-1, bt.hd)[heads + bt.kv:]
        if not no_q:
            got = qg[row].astype(np.float64).reshape(heads, bt.hd)
            assert np.all(np.abs(got - x[:heads]) <= tol[:heads]), row
    # and nothing else has changed
    assert np.array_equal(Kg.view(np.uint16), K.view(np.uint16))
    assert np.array_equal(to_host(bt.Vd).view(np.uint16), V.view(np.uint16))
    if not no_q:
        rows = {r for r, _, _ in bt.tokens()}
        rest = [r for r in range(bt.rows) if r not in rows]
        want = qkv[:, : heads * bt.hd] if in_place else np.full((bt.rows, heads * bt.hd), 5.0, np.float16)
        assert np.array_equal(to_host(q_out)[rest], want[rest])
    return qkv


@pytest.mark.parametrize("heads,kv,hd", HEADS + [(40, 40, 128)])
@pytest.mark.parametrize("single", [True, False])
def test_append(ctx, heads, kv, hd, single):
    rng = np.random.default_rng(1)
    lens = [(n, 1 if n else 0) for n in (1, 0, 16, 17, 300, 64)] if single else [(40, 40), (0, 0), (17, 1), (64, 0), (200, 33), (16, 16)]
    for page, norm, in_place in ((16, False, False), (64, True, True), (256, True, False)):
        gains = [rng.standard_normal(hd).astype(np.float16) if norm else None for _ in range(2)]
        bt = Batch(lens, kv, hd, page, seed=page, single=single, spare_rows=0 if single else 3)
        run_append(ctx, bt, heads, in_place=in_place, pad=8 if in_place else 0, gains=gains)


def test_append_many_rows(ctx):
    """Enough rows for the form that takes four tokens a workgroup, a last workgroup that is not full."""
    for hd in (64, 128):
        bt = Batch([(700, 600), (9, 9), (600, 520), (1, 1)], 1, hd, 16, seed=hd, spare_rows=2)
        run_append(ctx, bt, 2, gains=[np.ones(hd, np.float16)] * 2)


def test_append_options(ctx):
    """Positions of the caller's, far ones among them; another base; no queries; one norm without the other; zero rows."""
    heads, kv, hd = 4, 2, 64
    g = np.linspace(0.5, 2, hd).astype(np.float16)
    for kw in ({"theta": 500000.0}, {"no_q": True}, {"gains": (g, None)}, {"gains": (None, g), "eps": 0.0}, {"gains": (g, g), "eps": 0.5}):
        run_append(ctx, Batch([(40, 30), (5, 5)], kv, hd, 16, seed=3, gap=128), heads, **kw)
    bt = Batch([(40, 30), (5, 5)], kv, hd, 16, seed=3)
    run_append(ctx, bt, heads, pos=np.array([0, 1, 2 ** 20, 10 ** 6 + 7, 2 ** 30, -3] + list(range(29)), np.int32))
    none = Batch([(40, 0), (0, 0)], kv, hd, 16, seed=3)
    run_append(ctx, none, heads)
    zero = Batch([(4, 4)], kv, hd, 16, seed=3).upload()
    qkv = torch.zeros((4, 8 * hd), dtype=torch.float16, device="cuda")
    q = torch.ones((4, heads * hd), dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    gd = to_dev(g)
    ctx.paged_append(zero.cache, zero.batch, qkv, q, heads, q_gain=gd, k_gain=gd)
    ctx.synchronize()
    assert np.all(to_host(q) == 0)


@pytest.mark.parametrize("single", [True, False])
def test_append_reports_and_leaves_what_cannot_be_right(ctx, single):
    heads, kv, hd = 4, 2, 64
    bt = Batch([(100, 1), (40, 1), (50, 1)] if single else [(100, 30), (40, 20), (50, 50)], kv, hd, 16, seed=5, single=single)
    bt.table[0, 99 // 16] = 10 ** 6
    lens = list(bt.lens)
    bt.upload()
    bt.batch.kv_len[1] = -4
    rows = bt.rows
    qkv = to_dev(bt.rng.standard_normal((rows, 8 * hd)).astype(np.float16))
    q = torch.full((rows, heads * hd), 5.0, dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    ctx.paged_append(bt.cache, bt.batch, qkv, q, heads)
    ctx.synchronize()
    assert ctx.last_device_error() == B.AF_DEVERR_PAGED
    got, K = to_host(q), to_host(bt.Kd)
    for row, b, place in bt.tokens():
        gone = b == 1 or (b == 0 and place // 16 == 99 // 16)
        assert np.all(got[row] == 5.0) == gone
        if gone and b == 1:
            assert np.array_equal(K[bt.table[b, place // 16], :, place % 16], bt.K[bt.table[b, place // 16], :, place % 16])
    assert lens == bt.lens


# ---- together -------------------------------------------------------------------------------------------
def test_prompts_then_tokens(ctx):
    """A serving run: prompts of three requests, then tokens one at a time (with a captured step replayed as the
    sequences grow), then a mixed batch, all into one cache; every result against one pass over the whole sequence."""
    heads, kv, hd, page, cap = 8, 2, 64, 16, 12
    rng = np.random.default_rng(0)
    width = (heads + 2 * kv) * hd
    total = [150, 60, 97]
    x = [rng.standard_normal((n, width)).astype(np.float16) for n in total]
    done = [0, 0, 0]
    table = rng.permutation(3 * cap).reshape(3, cap).astype(np.int32)
    K, V = (torch.full((3 * cap, kv, page, hd), float("nan"), dtype=torch.float16, device="cuda") for _ in range(2))
    cache, tab, kv_len = B.PagedCache(K, V), to_dev(table), to_dev(np.zeros(3, np.int32))
    results = [np.zeros((n, heads * hd), np.float16) for n in total]
    g = np.ones(hd, np.float16)
    gd = to_dev(g)

    def call(batch, qkv, out):
        ctx.paged_append(cache, batch, qkv, qkv[:, : heads * hd], heads, q_gain=gd, k_gain=gd)
        ctx.paged_attention(cache, batch, qkv[:, : heads * hd], out, heads, window=64, n_sink=4)

    def ragged(counts):
        start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        for b in range(3):
            done[b] += counts[b]
        kv_len.copy_(to_dev(np.array(done, np.int32)))
        batch = B.PagedBatch(tab, kv_len, to_dev(start), int(start[-1]), max(counts))
        qkv = to_dev(np.concatenate([x[b][done[b] - counts[b]: done[b]] for b in range(3)]))
        out = torch.zeros((int(start[-1]), heads * hd), dtype=torch.float16, device="cuda")
        torch.cuda.synchronize()
        call(batch, qkv, out)
        ctx.synchronize()
        got = to_host(out)
        for b in range(3):
            results[b][done[b] - counts[b]: done[b]] = got[start[b]: start[b + 1]]

    ragged([70, 1, 33])
    ragged([20, 40, 1])
    single = B.PagedBatch(tab, kv_len)
    qkv = torch.zeros((3, width), dtype=torch.float16, device="cuda")
    out = torch.zeros((3, heads * hd), dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    graph = None
    for step in range(12):
        for b in range(3):
            done[b] += 1
        kv_len.copy_(to_dev(np.array(done, np.int32)))
        qkv.copy_(to_dev(np.stack([x[b][done[b] - 1] for b in range(3)])))
        torch.cuda.synchronize()
        if step < 2:
            call(single, qkv, out)
        else:
            if graph is None:
                ctx.capture_begin()
                call(single, qkv, out)
                graph = ctx.capture_end()
            ctx.graph_launch(graph)
        ctx.synchronize()
        got = to_host(out)
        for b in range(3):
            results[b][done[b] - 1] = got[b]
    ctx.graph_destroy(graph)
    ragged([total[b] - done[b] for b in range(3)])
    assert ctx.last_device_error() == 0

    whole = Batch([(n, n) for n in total], kv, hd, page, seed=1)
    whole.table = table
    whole.K, whole.V = to_host(K), to_host(V)
    q = np.zeros((sum(total), heads * hd), np.float16)
    qkv_all = np.concatenate(x)
    for row, (v, _) in append_ref(whole, qkv_all, heads, gains=(g, g)).items():
        q[row] = v[:heads].astype(np.float16).reshape(-1)
    ref = attend(whole, q, heads, 64, 4)
    got = np.concatenate(results).astype(np.float64).reshape(-1, heads, hd)
    for row, (o, mag) in ref.items():
        # as check(); and a query that fp32 rounds to the neighbouring fp16 shifts its scores (|k| some 8, 2^-11 of 1 each)
        assert np.all(np.abs(got[row] - o) <= 2.0 ** -11 * np.abs(o) + 2.0 ** -8 * mag), row


def test_two_contexts_and_a_stream_of_its_own(ctx):
    """Two contexts on streams of their own, the same cache: calls in flight at once, each with its own workspace."""
    heads, kv, hd = 8, 2, 128
    bt = Batch([(2000, 1), (900, 1)], kv, hd, 32, seed=12, single=True).upload()
    pr = Batch([(300, 200), (150, 150)], kv, hd, 32, seed=13).upload()
    other = B.Context(0)
    try:
        qa, qb = (to_dev((2 * b.rng.standard_normal((b.rows, heads * hd))).astype(np.float16)) for b in (bt, pr))
        oa, ob = torch.zeros_like(qa), torch.zeros_like(qb)
        torch.cuda.synchronize()
        for _ in range(5):
            ctx.paged_attention(bt.cache, bt.batch, qa, oa, heads)
            other.paged_attention(pr.cache, pr.batch, qb, ob, heads)
        ctx.synchronize()
        other.synchronize()
        check(to_host(oa), attend(bt, to_host(qa), heads), heads, hd)
        check(to_host(ob), attend(pr, to_host(qb), heads), heads, hd, weights16=True)
    finally:
        other.close()


def test_same_result_every_time(ctx):
    heads, kv, hd = 8, 2, 128
    for bt in (Batch([(5000, 1), (70, 1)], kv, hd, 16, seed=1, single=True), Batch([(400, 300), (600, 2)], kv, hd, 16, seed=1)):
        q, first = run(ctx, bt, heads)
        for _ in range(3):
            assert np.array_equal(run(ctx, bt, heads, q=q)[1].view(np.uint16), first.view(np.uint16))
