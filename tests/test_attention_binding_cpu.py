"""What the binding of the attention calls refuses before the library is asked. No GPU: host tensors stand for device ones, and
nothing is queued."""
import pytest
import torch

from paper_2005_04091_amd import attention as A


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
