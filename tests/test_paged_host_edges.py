"""Host side of the paged operators on the CPU, where their arguments have edges."""
import os
from types import SimpleNamespace

import pytest
import torch

from paper_2504_08378_amd import binding as B
from paper_2504_08378_amd import build
from test_paged_refusals import EINVAL, EWORKSPACE, _append, _attention


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(B.LIB_PATH):
        build.build(verbose=False)


def test_a_batch_without_rows_is_one(monkeypatch):
    """n_rows 0 without max_q_len: the bound is one row, as every call wants it."""
    monkeypatch.setattr(B, "_ptr", lambda t, *a: None if t is None else t.data_ptr())
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    s = B.PagedBatch(i32(3, 5), i32(3), i32(4), n_rows=0).struct
    batch = {n: getattr(s, n) for n, _ in B.PagedBatchStruct._fields_}
    for call in (_append, _attention):
        assert call(batch=batch) == EWORKSPACE   # past every check
    assert B.PagedBatch(i32(3, 5), i32(3), i32(4), n_rows=7).struct.max_q_len == 7
    assert B.PagedBatch(i32(3, 5), i32(3), i32(4), n_rows=7, max_q_len=4).struct.max_q_len == 4
    assert B.PagedBatch(i32(3, 5), i32(3)).struct.max_q_len == 1


def test_scales_at_the_end_of_the_range():
    """The kernels work with scale * log2(e): both have to be finite."""
    largest = float(torch.finfo(torch.float32).max)
    for scale in (largest, -largest, 2.5e38):
        assert _attention(scale=scale) == EINVAL
    for scale in (2.3e38, -2.3e38, 1e-38):
        assert _attention(scale=scale) == EWORKSPACE


def test_the_paged_layer_refuses_tensors_of_another_device():
    """As the single operators do: nothing of another device reaches a launch."""
    def tensor(device, n, dtype=torch.float16):
        return SimpleNamespace(is_cuda=True, dtype=dtype, get_device=lambda: device, numel=lambda: n, is_contiguous=lambda: True,
                               data_ptr=lambda: 4096)
    ctx = B.Context.__new__(B.Context)
    ctx.device, ctx._h = torch.device("cuda", 0), None
    cache = SimpleNamespace(index=0, head_dim=64, _ref=None)
    batch = SimpleNamespace(index=0, n_rows=2, _ref=None)
    cfg, w, sel, sets = B.LayerCfg(d_model=64), B.LayerWeights(), B.SelectCfg(), B.IdxSets()

    def call(**kw):
        t = {"hidden_in": tensor(0, 128), "hidden_out": tensor(0, 128), "union_n": None, **kw}
        ctx.decode_layer_batch_paged(cfg, w, t["hidden_in"], t["hidden_out"], cache, batch, sel, sets, union_n=t["union_n"])
    with pytest.raises(B.AfError):   # the library's own word for no context: the binding's checks are passed
        call()
    with pytest.raises(B.AfError):
        call(union_n=tensor(0, 4, torch.int32))
    for other in ({"hidden_in": tensor(1, 128)}, {"hidden_out": tensor(1, 128)}, {"union_n": tensor(1, 4, torch.int32)},
                  {"union_n": tensor(0, 3, torch.int32)}, {"hidden_in": tensor(0, 64)}):
        with pytest.raises(TypeError):
            call(**other)
