"""The paged operators where their batches have edges: what a row's weights are held to, whatever form forms it; tables with
entries that no token needs; batches without rows; padded batches, alone and through the layer; as many sequences as there
may be at width 128.  Against 64 bits, as in test_gpu_paged.py and with its tolerances."""
import numpy as np
import pytest
import torch

import synth_inputs as S
from paper_2504_08378_amd import binding as B
from paper_2504_08378_amd import model as M
from gpu_util import ctx, to_dev, to_host  # noqa: F401
from test_gpu_paged import Batch, attend, check, run
from test_gpu_paged_layer import Layer, _rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv,hd", [(4, 4, 64), (8, 2, 128), (20, 1, 64), (6, 2, 128)])
@pytest.mark.parametrize("lens", [[(2, 2), (40, 40), (77, 77), (33, 17)],             # a few tiles
                                  [(700, 300), (300, 1), (129, 129), (260, 7), (0, 0)],  # prompts and single tokens in one launch
                                  [(3000, 40), (900, 2)]])                            # keys in pieces
def test_weights_of_prompts_hold_more_than_fp16(ctx, heads, kv, hd, lens):
    """fp32 arithmetic and one rounding: 2^-17 of sum w|v| / sum w, where weights of 11 bits may be 2^-11 of it off."""
    for window, sinks, scale in ((0, 0, None), (50, 3, None), (0, 0, -0.3)):
        bt = Batch(lens, kv, hd, 16, seed=heads + window)
        kw = {} if scale is None else {"scale": scale}
        q, got = run(ctx, bt, heads, window=window, n_sink=sinks, **kw)
        check(got, attend(bt, q, heads, window, sinks, **kw), heads, hd)


def test_weights_of_prompts_in_fp16_where_the_caller_says_so(ctx):
    """AF_OPT_PAGED_F16_WEIGHTS: results within 2^-11 of sum w|v| / sum w more, and others than without it; single tokens as before."""
    heads, kv, hd = 8, 2, 128
    bt = Batch([(700, 300), (300, 1), (77, 77)], kv, hd, 16, seed=4)
    q, fine = run(ctx, bt, heads)
    ctx.set_option(B.AF_OPT_PAGED_F16_WEIGHTS, 1)
    try:
        _, coarse = run(ctx, bt, heads, q=q)
    finally:
        ctx.set_option(B.AF_OPT_PAGED_F16_WEIGHTS, 0)
    check(coarse, attend(bt, q, heads), heads, hd, weights16=True)
    assert not np.array_equal(coarse, fine) and np.array_equal(coarse[300], fine[300])
    assert np.array_equal(run(ctx, bt, heads, q=q)[1], fine)


@pytest.mark.parametrize("page", [16, 32])
@pytest.mark.parametrize("new", [1, 2, 40])
@pytest.mark.parametrize("window,sinks", [(100, 4), (100, 16), (100, 17), (100, 40), (31, 4), (33, 1), (16, 0), (1, 33)])
def test_pages_that_no_token_needs_may_be_gone(ctx, page, new, window, sinks):
    """Pages between the first tokens and the window, given back: entries that hold nothing are neither seen nor reported."""
    heads, kv, hd = 4, 2, 64
    lens = [(new + past, new) for past in (300, 47, 48, 63, 64, 130)]
    bt = Batch(lens, kv, hd, page, seed=window + sinks, single=new == 1)
    gone = 0
    for b, (n, q) in enumerate(lens):
        j = np.arange(n)
        seen = (j > n - q - window) | (j < sinks)
        for e in range(-(-n // page)):
            if not np.any(seen[e * page: (e + 1) * page]):
                bt.table[b, e] = -1
                gone += 1
    assert gone
    q, got = run(ctx, bt, heads, window=window, n_sink=sinks)
    check(got, attend(bt, q, heads, window, sinks), heads, hd)


@pytest.mark.parametrize("seqs", [65, 1024])
def test_many_sequences_and_a_prompt_at_width_128(ctx, seqs):
    """One launch for single tokens, prompts and empty ranges, its look-up table in LDS beside the tiles of the wider heads."""
    heads, kv, hd = 4, 2, 128
    rng = np.random.default_rng(seqs)
    lens = [(int(n), int(min(n, q))) for n, q in zip(rng.integers(1, 40, seqs), rng.choice([0, 1, 2, 12], seqs))]
    lens[seqs // 2] = (700, 200)
    for window, sinks in ((0, 0), (20, 3)):
        bt = Batch(lens, kv, hd, 16, seed=seqs, spare_rows=3)
        q, got = run(ctx, bt, heads, window=window, n_sink=sinks)
        check(got, attend(bt, q, heads, window, sinks), heads, hd, untouched=5.0)


@pytest.mark.parametrize("heads,kv,hd", [(8, 2, 64), (32, 8, 128)])
def test_a_chunk_behind_a_long_past_among_single_tokens(ctx, heads, kv, hd):
    """A serving step of chunked prompts: one request's next 100 tokens behind 2500, the others one token each."""
    lens = [(1 + 37 * i % 300, 1) for i in range(40)]
    lens[23] = (2600, 100)
    bt = Batch(lens, kv, hd, 16, seed=heads)
    q, got = run(ctx, bt, heads)
    check(got, attend(bt, q, heads), heads, hd)


# ---- padded batches through the layer --------------------------------------------------------------------
def _hidden(shape, n, first=0):
    scales = S.channel_scales(0, shape.d_model, shape.name)
    return np.stack([S.activation(0, scales, "hidden", first + i) for i in range(n)])


def _past(ctx, shape, seqs, lens):
    """A book of pages whose sequences hold random keys and values."""
    kv = M.PagedKv(ctx, shape, 1, n_pages=60, page_tokens=16, max_seqs=seqs, max_tokens=160)
    kv.extend(lens)
    g = torch.Generator(device="cuda").manual_seed(7)
    for t in (kv.layers[0].k_pages, kv.layers[0].v_pages):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda").half())
    return kv


@pytest.mark.parametrize("shape_name", ["tiny_gqa", "tiny_hd128"])
@pytest.mark.parametrize("fill", [0.5, np.inf, np.nan])
def test_layer_rows_behind_the_last_sequence(ctx, shape_name, fill):
    """Spare rows of a ragged batch hold `fill`, the layer's own tensors what an earlier call of NaN has left in them: the rows
    with a token are what they are without all that."""
    shape = S.MODEL_SHAPES[shape_name]
    lay = Layer(ctx, shape)
    stale = _past(ctx, shape, 8, [3] * 8)
    lay.run(np.full((8, shape.d_model), np.nan, np.float16), stale.layers[0], stale.extend([1] * 8))
    assert torch.isnan(ctx.layer_tap(2, 8 * shape.n_heads * shape.head_dim)).all()
    lens, counts = [37, 90, 5], [2, 0, 1]
    kv = _past(ctx, shape, 3, lens)
    got = kv.extend(counts)
    batch = B.PagedBatch(kv.table, kv.kv_len, got.q_start, n_rows=7, max_q_len=2)
    H = np.concatenate([_hidden(shape, 3), np.full((4, shape.d_model), fill, np.float16)])
    out = lay.run(H, kv.layers[0], batch)
    for row, b, place in ((0, 0, 37), (1, 0, 38), (2, 2, 5)):
        K, V = _rows(kv.layers[0], kv.table, b, place + 1)
        lay.check(row, 7, H[row], out[row], K, V, place)


def test_layer_replayed_with_a_released_sequence(ctx):
    """A captured step of one token each goes on when a request has ended: its row, with NaN in it, has no token, and the
    others' results are right; then another request takes the place."""
    shape = S.MODEL_SHAPES["tiny_gqa"]
    lay = Layer(ctx, shape)
    kv = _past(ctx, shape, 3, [20, 33, 60])
    hin = torch.zeros((3, shape.d_model), dtype=torch.float16, device="cuda")
    out = torch.zeros_like(hin)
    cfg, w, sel, sets = M.layer_cfg(shape), lay.dev.struct(), M.select_cfg(B.AF_SEL_TOPK, lay.ks), lay.sets(3)
    batch = B.PagedBatch(kv.table, kv.kv_len)
    torch.cuda.synchronize()
    ctx.capture_begin()
    ctx.decode_layer_batch_paged(cfg, w, hin, out, kv.layers[0], batch, sel, sets, window=40, n_sink=2)
    graph = ctx.capture_end()

    def step(counts, first):
        kv.extend(counts)
        H = _hidden(shape, 3, first)
        for b, c in enumerate(counts):
            if c == 0:
                H[b] = np.nan
        hin.copy_(to_dev(H))
        torch.cuda.synchronize()
        ctx.graph_launch(graph)
        ctx.synchronize()
        assert ctx.last_device_error() == 0
        got = to_host(out)
        for b, c in enumerate(counts):
            if c:
                K, V = _rows(kv.layers[0], kv.table, b, kv.lens[b])
                lay.check(b, 3, H[b], got[b], K, V, kv.lens[b] - 1, 40, 2)
    try:
        step([1, 1, 1], 0)
        kv.release(1)
        step([1, 0, 1], 3)
        step([1, 0, 1], 6)
        kv.extend([0, 8, 0])        # the next request's first tokens are in the cache already
        step([1, 1, 1], 9)
    finally:
        ctx.synchronize()
        ctx.graph_destroy(graph)


def test_calls_without_rows(ctx):
    """Zero rows, with and without sequences that have tokens: nothing is launched, nothing refused."""
    bt = Batch([(40, 0), (0, 0)], 2, 64, 16, seed=3).upload()
    batch = B.PagedBatch(bt.batch.page_table, bt.batch.kv_len, bt.batch.q_start, n_rows=0)
    none = torch.empty((0, 4 * 64), dtype=torch.float16, device="cuda")
    before = bt.Kd.clone()
    ctx.paged_append(bt.cache, batch, torch.empty((0, 8 * 64), dtype=torch.float16, device="cuda"), none, 4)
    ctx.paged_attention(bt.cache, batch, none, none.clone(), 4)
    ctx.synchronize()
    assert ctx.last_device_error() == 0 and torch.equal(bt.Kd.view(torch.int16), before.view(torch.int16))
