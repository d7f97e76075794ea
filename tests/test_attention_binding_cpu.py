"""What the attention calls refuse: the binding before the library is asked, and the library. No GPU: host tensors stand for
device ones, and nothing is queued."""
import pytest
import torch

from paper_2005_04091_amd import attention as A

P = 4096  # an aligned address; nothing is read there


def host_batch(B=3, nb=4, block=16, q_block=1):
    """A batch whose tensors lie on the host."""
    batch = A.CacheBatch.__new__(A.CacheBatch)
    batch.device = torch.device("cpu")
    batch.table, batch.kv_len, batch.q_start = torch.zeros((B, nb), dtype=torch.int32), torch.ones(B, dtype=torch.int32), None
    batch.sequences, batch.max_blocks, batch.block, batch.q_block, batch.tokens, batch.rows = B, nb, block, q_block, B, B
    batch._fields = (B, block, nb, q_block, B, nb, batch.table.data_ptr(), batch.kv_len.data_ptr(), None)
    batch._last = (0, None)
    return batch


def test_empty_lists_are_refused():
    """Lists without entries list nothing; without an address they would stand for every block."""
    q, cache = torch.zeros(3, 2, 64), torch.zeros(5, 2, 16, 64)
    with pytest.raises(A.SpconvError) as e:
        A.spconv_block_attention(q, cache, cache.clone(), host_batch(), torch.zeros((3, 2, 0), dtype=torch.int32))
    assert e.value.code == A.SPCONV_EINVAL


def test_tensors_that_require_grad_are_refused():
    """Their gradients would be lost without a word."""
    batch, q, cache = host_batch(), torch.zeros(3, 2, 64), torch.zeros(5, 2, 16, 64)
    grad = lambda t: t.clone().requires_grad_(True)
    sums, freq, scores = torch.zeros(5, 2, 64), torch.ones(4, dtype=torch.float64), torch.zeros(3, 2, 4)
    for call in (lambda: A.spconv_cache_append(grad(q), q, cache, cache, batch), lambda: A.spconv_cache_append(q, grad(q), cache, cache, batch),
                 lambda: A.spconv_cache_append(q, q, grad(cache), cache, batch), lambda: A.spconv_block_scores(grad(q), sums, batch),
                 lambda: A.spconv_cache_append(q, q, cache, cache, batch, freq=grad(freq)), lambda: A.spconv_block_scores(q, grad(sums), batch), lambda: A.spconv_select_blocks(grad(scores), batch, 4),
                 lambda: A.spconv_block_attention(grad(q), cache, cache, batch), lambda: A.spconv_block_attention(q, grad(cache), cache, batch),
                 lambda: A.spconv_block_attention(q, cache, grad(cache), batch)):
        with pytest.raises(ValueError, match="requires grad"):
            call()
    x = grad(q)
    with torch.no_grad():
        assert A._rows(x, "x", x.dtype, x.shape, x.device)[0] == A._whole(x, "x", x.dtype, x.shape, x.device) == x.data_ptr()
    assert A._rows(x.detach(), "x", x.dtype, x.shape, x.device)[0] == x.data_ptr()


def test_what_is_no_tensor_is_a_type_error():
    batch, q, cache = host_batch(), torch.zeros(3, 2, 64), torch.zeros(5, 2, 16, 64)
    for call in (lambda: A.spconv_cache_append(None, q, cache, cache, batch), lambda: A.spconv_cache_append(q, q, [1], cache, batch),
                 lambda: A.spconv_block_scores([[1.0]], cache[:, :, 0], batch), lambda: A.spconv_block_scores(q, None, batch),
                 lambda: A.spconv_select_blocks(None, batch, 4), lambda: A.spconv_block_attention("q", cache, cache, batch),
                 lambda: A.spconv_block_attention(q, None, cache, batch), lambda: A.spconv_block_attention(q, cache, cache, batch, [[[0]]])):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError, match="tokens, heads, dim"):
        A.spconv_block_attention(q[0], cache, cache, batch)
    with pytest.raises(ValueError, match="pages, heads, block, dim"):
        A.spconv_block_attention(q, cache[0], cache, batch)


def test_a_workspace_of_an_unknown_type_is_a_type_error():
    with pytest.raises(TypeError):
        A.spconv_attention_workspace(torch.float64, host_batch(), 8, 2, 64)
    assert A.spconv_attention_workspace(torch.float16, host_batch(), 8, 2, 64) == 0


def test_sizes_are_whole_numbers(monkeypatch):
    """Also where the library's answer for the equal number is remembered."""
    monkeypatch.setattr(A, "_device", lambda t, name: t.device)
    table, kv, start = torch.zeros((2, 4), dtype=torch.int32), torch.ones(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    assert A.CacheBatch(table, kv, 16, start, 40, 8).rows == 40 // 8 + 2
    for bad in [dict(block=16.0), dict(q_block=8.0), dict(tokens=40.0)]:
        with pytest.raises(TypeError):
            A.CacheBatch(table, kv, **{**dict(block=16, q_start=start, tokens=40, q_block=8), **bad})
    args = dict(q_heads=8, heads=2, dim=64, keep=4)
    A.spconv_attention_workspace(torch.float16, host_batch(), **args)
    for name in args:
        with pytest.raises(TypeError):
            A.spconv_attention_workspace(torch.float16, host_batch(), **{**args, name: float(args[name])})


def test_a_scale_past_the_range_is_refused():
    """The kernels count in powers of two: a scale whose product with log2(e) is infinite would make every output NaN."""
    def attend(scale):
        return A._lib.spconv_block_attention(2, A.spconv_batch(2, 64, 8, 1, 10, 20, 8, P, P, P), P, 4096, 128, 32, 8, 128, P, P, scale, P, P,
                                             4, P + 64, 4096, 128, None, P, 1 << 40, None)
    for scale in (3e38, -3e38, float("inf"), float("nan")):
        assert attend(scale) == A.SPCONV_EINVAL
