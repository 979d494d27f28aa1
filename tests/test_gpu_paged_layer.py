"""af_decode_layer_batch_paged: the batched layer over a paged cache.  Every token is judged stage by stage against the
oracle's operators on the bits the GPU fed into each stage (as the batched layer over caches of their own is), with its
queries rounded to fp16 between rotation and attention; and a run of steps through model.PagedKv as a serving loop makes them."""
import numpy as np
import pytest
import torch

import synth_inputs as S
from oracle import activeflow_oracle as O
from paper_2504_08378_amd import binding as B
from paper_2504_08378_amd import model as M
from gpu_util import TAP_NAMES, ctx, teacher_forced_layer_errors, to_dev, to_host  # noqa: F401

pytestmark = pytest.mark.gpu
TOL = 2e-3


def _widths(shape):
    return (shape.d_model, shape.n_heads * shape.head_dim, shape.d_model, shape.d_ffn)


class Layer:
    def __init__(self, ctx, shape, seed=0):
        self.ctx, self.shape = ctx, shape
        self.w = S.layer_weights(seed, shape, 0)
        self.dev = M.DeviceLayer(ctx, shape, self.w)
        self.ks = tuple(O.keep_count(n, 50) for n in _widths(shape))

    def sets(self, rows):
        self.idx = [torch.zeros((rows, n), dtype=torch.int32, device="cuda") for n in _widths(self.shape)]
        self.cnt = [torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(4)]
        s = B.IdxSets()
        for p in range(4):
            s.idx[p], s.count[p] = self.idx[p].data_ptr(), self.cnt[p].data_ptr()
        return s

    def run(self, H, cache, batch, **kw):
        sets = self.sets(len(H))
        hin = to_dev(H)
        out = torch.zeros_like(hin)
        torch.cuda.synchronize()
        self.ctx.decode_layer_batch_paged(M.layer_cfg(self.shape), self.dev.struct(), hin, out, cache, batch,
                                          M.select_cfg(B.AF_SEL_TOPK, self.ks), sets, **kw)
        self.ctx.synchronize()
        assert self.ctx.last_device_error() == 0
        return to_host(out)

    def check(self, row, n_rows, h_in, h_out, K, V, place, window=0, sinks=0, weights16=False):
        """Row `row` of the last call; K, V [kv][tokens][hd] on the host with the new token's row in."""
        sh = self.shape
        d, f, hd, nh, nkv = sh.d_model, sh.d_ffn, sh.head_dim, sh.n_heads, sh.n_kv_heads
        sizes = (d, (nh + 2 * nkv) * hd, nh * hd, d, d, 2 * f, f)
        taps = {n: to_host(self.ctx.layer_tap(i, s * n_rows)).reshape(n_rows, s)[row] for i, (n, s) in enumerate(zip(TAP_NAMES, sizes))}
        idx = [to_host(self.idx[p])[row, : int(self.cnt[p][row])] for p in range(4)]
        cfg = O.LayerCfg(d, nh, nkv, hd, f)
        sel = O.SelectCfg(O.SEL_TOPK, self.ks)
        pad = lambda a: np.concatenate([a, np.zeros_like(a[:, :1])], 1)
        errs, own = teacher_forced_layer_errors(O, cfg, self.w, h_in, pad(K), pad(V), place, place, taps, h_out, idx, sel)
        q = O.round_f16(O.rope(taps["qkv"][: nh * hd].reshape(nh, hd), place, 10000.0))
        k = O.round_f16(O.rope(taps["qkv"][nh * hd: (nh + nkv) * hd].reshape(nkv, hd), place, 10000.0))
        assert O.rel_err(K[:, place], k) <= TOL
        assert np.array_equal(V[:, place], taps["qkv"][(nh + nkv) * hd:].reshape(nkv, hd))
        j = np.arange(place + 1)
        j = j if not window else j[(j > place - window) | (j < sinks)]
        # Attention: one rounding of the result (half of 2^-10 of it), the fp32 arithmetic (2^-17 of sum w|v|, some 64 roundings)
        # and, where a prompt's weights are held in fp16, half of 2^-10 of each.  The queries are known to the oracle up to the
        # rounding of values that fp32 (2^-20 of the pair's length) may put on the other side of the border between two fp16
        # values: those change a score by up to `shift`, every weight by a factor of e^(+-shift), the result by 2 shift sum w|v|.
        rep, q64 = nh // nkv, O.rope(taps["qkv"][: nh * hd].reshape(nh, hd), place, 10000.0).astype(np.float64)
        eps = 2.0 ** -20 * np.tile(np.hypot(q64[:, : hd // 2], q64[:, hd // 2:]), 2)
        open_ = np.abs(O.round_f16(q64 + eps).astype(np.float64) - O.round_f16(q64 - eps))
        Kj, Vj = (np.repeat(x[:, j].astype(np.float64), rep, 0) for x in (K, V))
        shift = np.einsum("hd,hjd->hj", open_, np.abs(Kj)).max(1)[:, None] / np.sqrt(hd)
        s_ = np.einsum("hd,hjd->hj", q.astype(np.float64), Kj) / np.sqrt(hd)
        w_ = np.exp(s_ - s_.max(1, keepdims=True))
        w_ /= w_.sum(1, keepdims=True)
        att, mag = (np.einsum("hj,hjd->hd", w_, x) for x in (Vj, np.abs(Vj)))
        tol = 2.0 ** -11 * np.abs(att) + 2.0 ** -25 + mag * (2.0 ** -17 + (2.0 ** -11 if weights16 else 0) + 2 * shift)
        assert np.all(np.abs(taps["attn"].astype(np.float64).reshape(nh, hd) - att) <= tol)
        del errs["attn"]
        assert max(errs.values()) <= TOL, errs
        assert all(np.array_equal(idx[p], own[p]) for p in range(4))


def _rows(cache, table, b, n):
    """The first n tokens' rows of sequence b: K, V [kv][n][hd]."""
    page = cache.k_pages.shape[2]
    pg = to_host(table)[b, np.arange(n) // page]
    return [to_host(t)[pg, :, np.arange(n) % page].transpose(1, 0, 2) for t in (cache.k_pages, cache.v_pages)]


@pytest.mark.parametrize("shape_name", ["tiny_gqa", "tiny_hd128"])
@pytest.mark.parametrize("seqs", [1, 3, 8])
def test_single_tokens_of_their_own_lengths(ctx, shape_name, seqs):
    shape = S.MODEL_SHAPES[shape_name]
    lay = Layer(ctx, shape)
    kv = M.PagedKv(ctx, shape, 1, n_pages=60, page_tokens=16, max_seqs=seqs, max_tokens=160)
    lens = [(7 + 41 * b) % 130 for b in range(seqs)]
    kv.extend(lens)                       # a past of random keys and values
    g = torch.Generator(device="cuda").manual_seed(5)
    with torch.cuda.stream(ctx.stream):
        for t in (kv.layers[0].k_pages, kv.layers[0].v_pages):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda").half())
    batch = kv.extend([1] * seqs)
    H = np.stack([S.activation(0, S.channel_scales(0, shape.d_model, shape.name), "hidden", b) for b in range(seqs)])
    out = lay.run(H, kv.layers[0], batch)
    for b in range(seqs):
        K, V = _rows(kv.layers[0], kv.table, b, lens[b] + 1)
        lay.check(b, seqs, H[b], out[b], K, V, lens[b])


def test_agrees_with_caches_of_their_own(ctx):
    """The same tokens, keys and values through af_decode_layer_batch: up to the queries' rounding."""
    shape = S.MODEL_SHAPES["tiny_hd128"]
    lay = Layer(ctx, shape)
    lens, cap = [33, 90, 5, 64], 128
    kv = M.PagedKv(ctx, shape, 1, n_pages=40, page_tokens=16, max_seqs=4, max_tokens=cap)
    kv.extend(lens)
    caches = [S.kv_cache(1, shape.n_kv_heads, cap, shape.head_dim, n, shape.name, b) for b, n in enumerate(lens)]
    for b, (K, V) in enumerate(caches):
        for j in range(lens[b]):
            page, slot = kv.pages[b][j // 16], j % 16
            kv.layers[0].k_pages[page, :, slot] = to_dev(K[:, j])
            kv.layers[0].v_pages[page, :, slot] = to_dev(V[:, j])
    H = np.stack([S.activation(0, S.channel_scales(0, shape.d_model, shape.name), "hidden", b) for b in range(4)])
    got = lay.run(H, kv.layers[0], kv.extend([1] * 4))
    hin, out = to_dev(H), torch.zeros((4, shape.d_model), dtype=torch.float16, device="cuda")
    Kd, Vd = [to_dev(K) for K, _ in caches], [to_dev(V) for _, V in caches]
    torch.cuda.synchronize()
    ctx.decode_layer_batch(M.layer_cfg(shape), lay.dev.struct(), hin, out, Kd, Vd, lens, cap, lens,
                           M.select_cfg(B.AF_SEL_TOPK, lay.ks), lay.sets(4))
    ctx.synchronize()
    assert O.rel_err(got, to_host(out).astype(np.float64), 1.0) <= 2 * TOL


def test_serving_run(ctx):
    """Two layers, three requests: prompts in pieces of up to eight tokens, then single tokens with a window, a request that ends
    and another that takes its pages, and a captured step that stays valid while the sequences grow."""
    shape = S.MODEL_SHAPES["tiny_gqa"]
    lays = [Layer(ctx, shape, 0), Layer(ctx, shape, 1)]
    kv = M.PagedKv(ctx, shape, 2, n_pages=24, page_tokens=16, max_seqs=3, max_tokens=112)
    rng = np.random.default_rng(2)
    scales = S.channel_scales(0, shape.d_model, shape.name)
    n_act = [0]

    def hidden(n):
        n_act[0] += n
        return np.stack([S.activation(0, scales, "hidden", n_act[0] + i) for i in range(n)])

    def step(counts, check=True):
        before = list(kv.lens)
        batch = kv.extend(counts)
        H = hidden(sum(counts))
        for l, lay in enumerate(lays):
            out = lay.run(H, kv.layers[l], batch, window=40, n_sink=2)
            row = 0
            for b, c in enumerate(counts):
                for i in range(c):
                    if check and rng.random() < 0.5:
                        K, V = _rows(kv.layers[l], kv.table, b, before[b] + i + 1)
                        lay.check(row, len(H), H[row], out[row], K, V, before[b] + i, 40, 2,
                                  weights16=c > 1 and c * shape.n_heads // shape.n_kv_heads > 16)
                    row += 1
            H = out
        return H

    step([8, 0, 0]); step([4, 3, 1]); step([0, 5, 2]); step([1, 1, 6])
    for _ in range(45):
        step([1, 1, 1], check=False)
    step([1, 1, 1])
    kv.release(1)
    assert len(kv.free_pages) == 24 - len(kv.pages[0]) - len(kv.pages[2])
    step([0, 7, 1]); step([1, 1, 1])

    # a captured step: two layers, replayed while the lengths grow
    batch = B.PagedBatch(kv.table, kv.kv_len)
    hin = torch.zeros((3, shape.d_model), dtype=torch.float16, device="cuda")
    mid, out = torch.zeros_like(hin), torch.zeros_like(hin)
    cfg, sel = M.layer_cfg(shape), M.select_cfg(B.AF_SEL_TOPK, lays[0].ks)
    s0, s1 = lays[0].sets(3), lays[1].sets(3)
    w0, w1 = lays[0].dev.struct(), lays[1].dev.struct()

    def call():
        ctx.decode_layer_batch_paged(cfg, w0, hin, mid, kv.layers[0], batch, sel, s0, window=40, n_sink=2)
        ctx.decode_layer_batch_paged(cfg, w1, mid, out, kv.layers[1], batch, sel, s1, window=40, n_sink=2)
    torch.cuda.synchronize()
    ctx.capture_begin()
    call()
    graph = ctx.capture_end()
    for _ in range(20):
        kv.extend([1, 1, 1])
        hin.copy_(to_dev(hidden(3)))
        torch.cuda.synchronize()
        ctx.graph_launch(graph)
        ctx.synchronize()
        got = to_host(out)
        out.zero_()
        torch.cuda.synchronize()
        call()                            # the same step again, eagerly: the same bits
        ctx.synchronize()
        assert np.array_equal(to_host(out).view(np.uint16), got.view(np.uint16))
    ctx.graph_destroy(graph)
    assert ctx.last_device_error() == 0


def test_what_it_refuses(ctx):
    shape = S.MODEL_SHAPES["tiny_gqa"]
    lay = Layer(ctx, shape)
    kv = M.PagedKv(ctx, shape, 1, n_pages=8, page_tokens=16, max_seqs=2, max_tokens=48)
    batch = kv.extend([1, 1])
    H = np.zeros((2, shape.d_model), np.float16)
    for kw in ({"window": -1}, {"n_sink": -1}):
        with pytest.raises(B.AfError):
            lay.run(H, kv.layers[0], batch, **kw)
    other = M.PagedKv(ctx, S.MODEL_SHAPES["tiny_hd128"], 1, n_pages=4, page_tokens=16, max_seqs=2, max_tokens=16)
    with pytest.raises(B.AfError) as e:
        lay.run(H, other.layers[0], batch)
    assert e.value.status == -3
    with pytest.raises(B.AfError):        # more rows than the layer takes
        lay.run(np.zeros((9, shape.d_model), np.float16), kv.layers[0], kv.extend([9, 0]))
    with pytest.raises(TypeError):
        lay.run(H[:1], kv.layers[0], batch)
    with pytest.raises(MemoryError):
        M.PagedKv(ctx, shape, 1, 1, 16, 1, 48).extend([17])
    with pytest.raises(ValueError):
        M.PagedKv(ctx, shape, 1, 8, 16, 1, 48).extend([49])
