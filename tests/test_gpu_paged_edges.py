"""The paged operators where their batches have edges: what a row's weights are held to, whatever form forms it; tables with
entries that no token needs; batches without rows; padded batches, alone and through the layer; as many sequences as there
may be at width 128.  Against 64 bits, as in test_gpu_paged.py and with its tolerances."""
import numpy as np
import pytest
import torch

from paper_2504_08378_amd import binding as B
from gpu_util import ctx, to_dev, to_host  # noqa: F401
from test_gpu_paged import Batch, attend, check, run

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
