"""What the extension leaves to Python of the paged calls, and where they may run."""
import pytest
import torch

from paper_2601_20499_amd import binding as df
from tests import paged_util as pu


def batch():
    return pu.Batch(0, [20, 5], [3, 4], [(0, pu.FULL), (4, 16)], G=2, d=64, device="cpu")


def test_what_is_not_ordinary_is_left_to_python():
    native = df._marshal()
    b = batch()
    cache, q, slots, one = b.cache(df), b.q, torch.zeros(7, 2, dtype=torch.int64), torch.zeros(1, dtype=torch.int32)
    assert native.page_map(cache, b.cu, slots, one, None, b.length, b.n_free, None) is None             # not on a GPU
    assert native.paged_append(cache, b.k_new, b.v_new, slots, None) is None
    assert native.paged_attn(q, None, None, cache, b.cu, q, 0.125, 1, None, None, None, None) is None
    for call, n in ((native.page_map, 8), (native.paged_append, 5), (native.paged_attn, 12)):
        assert call() is None and call(*[object()] * n) is None and call(*[None] * n) is None and call(*[None] * (n + 1)) is None
    with pytest.raises(TypeError):
        native.setup_paged(1)
    with pytest.raises(ValueError):
        native.setup_paged(0, 0, 0)


def test_a_cache_of_another_gpu_is_refused(monkeypatch):
    b = batch()
    cache = b.cache(df)
    cache.device = torch.device("cuda", 1)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    slots, status = torch.zeros(7, 2, dtype=torch.int64), torch.zeros(1, dtype=torch.int32)
    for call in (lambda: df.df_page_map(cache, b.cu, slots, status), lambda: df.df_paged_append(cache, b.k_new, b.v_new, slots),
                 lambda: df.df_paged_attn(b.q, None, None, cache, b.cu, b.q, 0.125)):
        with pytest.raises(ValueError, match="not on the current GPU"):
            call()


def test_a_scale_that_leaves_32_bits_is_refused():
    """The kernels work with the scale times log2(e)."""
    from tests import test_paged_abi as abi
    for scale, code in ((3e38, df.DF_ERR_RANGE), (2e38, df.DF_ERR_WORKSPACE)):
        assert abi._calls(df, abi._cache(df), softmax_scale=scale, workspace=None)[2]() == code


def test_batches_of_more_rows_than_a_launch_has_threads_are_refused():
    from tests import test_paged_abi as abi
    wide = abi._cache(df, H_kv=64, cap_stride=0)
    assert abi._calls(df, wide, total_new=1 << 30)[0]() == df.DF_ERR_RANGE and abi._calls(df, wide, total_new=1 << 28)[1]() == df.DF_ERR_RANGE


def test_a_workspace_that_is_not_what_it_counts_is_refused():
    b = batch()
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1 << 26), torch.zeros(64, 64)[:, ::2]):
        with pytest.raises(ValueError, match="workspace"):
            df.df_paged_attn(b.q, None, None, b.cache(df), b.cu, b.q, 0.125, workspace=ws)
