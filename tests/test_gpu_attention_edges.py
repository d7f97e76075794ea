"""GPU tests of the attention calls where sizes and values meet that a step seldom has at once: rows of several tokens for
single tokens, values that are not finite beside keys that are masked, far positions. The forms and bounds are
attention_oracle.py's; infinities and NaN have to come out as themselves."""
import numpy as np
import pytest
import torch

import attention_oracle as O
import test_gpu_attention as T
from paper_2005_04091_amd import attention as A

pytestmark = pytest.mark.gpu
TYPES, DEV, f64, normal, Setup, random_lists = T.TYPES, T.DEV, T.f64, T.normal, T.Setup, T.random_lists


def near(got, want, bound, what=""):
    """Finite numbers within the bound; infinities of the same sign and NaN where those are due, and nowhere else."""
    got = f64(got) if isinstance(got, torch.Tensor) else got
    odd = ~np.isfinite(want)
    with np.errstate(invalid="ignore"):
        fine = np.where(odd, (got == want) | (np.isnan(got) & np.isnan(want)), np.abs(got - want) <= bound)
    assert fine.all(), (what, int((~fine).sum()), got[~fine][:4], want[~fine][:4], np.argwhere(~fine)[:4])


def check_attention(s, q, heads, blocks=None, counts=None, scale=None):
    """Outputs between guards, against the formula."""
    dev = lambda a: None if a is None else torch.from_numpy(a).to(DEV)
    n, D = q.shape[0], q.shape[2]
    out = torch.full((n + 256, *q.shape[1:]), 3.0, dtype=q.dtype, device=DEV)
    lse = torch.full((n + 256, q.shape[1]), 3.0, device=DEV)
    A.spconv_block_attention(q, s.k, s.v, s.batch, dev(blocks), dev(counts), scale, out[128:-128], lse[128:-128])
    wo, wl, bo, bl = O.attention(s.rows, f64(q), f64(s.k), f64(s.v), s.table, s.block, D ** -0.5 if scale is None else scale, blocks,
                                 counts, q.dtype)
    mine = np.zeros(n + 256, bool)
    for _, toks, _ in s.rows.of.values():
        mine[[t + 128 for t in toks]] = True
    assert (f64(out)[~mine] == 3.0).all() and (f64(lse)[~mine] == 3.0).all()
    some = mine[128:-128]
    near(f64(out)[mine], wo[some], bo[some], "out")
    near(f64(lse)[mine], wl[some], bl[some], "lse")
    return out[128:-128], lse[128:-128]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,q_block,group", [(1, 2, 4), (3, 2, 1), (64, 16, 4), (70, 4, 20), (5, 128, 4), (200, 8, 2), (17, 16, 8)])
def test_single_tokens_in_rows_of_several(dtype, B, q_block, group):
    """Without q_start sequence b is token b of row b/q_block + b; the rows between and behind have no tokens."""
    rng = np.random.default_rng(B * 131 + q_block)
    s = Setup(rng, [1] * B, rng.integers(0, 300, B), 16, 2, 64, dtype, q_block, decode=True)
    q = normal(rng, (B, 2 * group, 64), dtype)
    all_keys = check_attention(s, q, 2)
    blocks, counts = random_lists(rng, s, 2, 6)
    check_attention(s, q, 2, blocks, counts)
    sums = normal(rng, (s.pages, 2, 64), torch.float32, 3.0)
    want, bound = O.scores(s.rows, f64(q), f64(sums), s.table, s.kv, 16, 2)
    got = A.spconv_block_scores(q, sums, s.batch)
    near(got, want, bound, "scores")
    keep = 2 + -(-(q_block - 1) // 16)
    wb, wc = O.select(s.rows, f64(got), 16, keep, 1, 1)
    blocks, counts = A.spconv_select_blocks(got, s.batch, keep)
    assert np.array_equal(blocks.cpu().numpy(), wb) and np.array_equal(counts.cpu().numpy(), wc)
    check_attention(s, q, 2, wb, wc)
    # Nothing of it depends on q_block where there are no lists.
    one = A.CacheBatch(s.batch.table, s.batch.kv_len, 16)
    assert all(torch.equal(a, b) for a, b in zip(all_keys, A.spconv_block_attention(q, s.k, s.v, one, lse=True)))
    # The append: a token's key and value to its sequence's newest slot.
    k, v = (normal(rng, (B, 2, 64), dtype) for _ in range(2))
    kc, vc, sums = s.k.clone(), s.v.clone(), torch.zeros((s.pages, 2, 64), device=DEV)
    A.spconv_cache_append(k, v, kc, vc, s.batch, sums)
    want_k, want_v = s.k.clone(), s.v.clone()
    for b in range(B):
        if s.kv[b]:
            at = int(s.table[b, (s.kv[b] - 1) // 16]), slice(None), int(s.kv[b] - 1) % 16
            want_k[at], want_v[at] = k[b], v[b]
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("q_block", [1, 3, 16])
def test_values_that_are_not_finite_beside_masked_keys(dtype, dim, q_block):
    """Infinities and NaN of values that a query sees come out, also where the block beside theirs in a tile is seen in part,
    is no block, has no page, or where the list ends behind theirs; those that it does not see stay out."""
    rng = np.random.default_rng(dim + q_block)
    s = Setup(rng, [6, 21], [90, 120], 16, 2, dim, dtype, q_block, extra_cols=1)
    s.table[1, 4] = -1
    s.make()
    for b in range(2):
        for pos, d, x in [(70, 1, "nan"), (65, 3, "inf"), (74, dim - 1, "-inf"), (10, 9, "inf"), (85, 11, "nan"), (87, 13, "-inf"),
                          (50, 5, "inf"), (30, 7, "nan")]:
            page = int(s.table[b, pos // 16])
            if page >= 0:
                s.v[page, pos % 2, pos % 16, d] = float(x)
    q = normal(rng, (s.tokens, 8, dim), dtype)
    check_attention(s, q, 2)
    lists = np.array([[4, 5, -1], [0, -1, 5], [4, -1, -1], [1, 5, 2], [3, 0, 4], [-1, 3, 4], [5, 4, 3], [4, 3, 0], [6, 7, 2]], np.int32)
    blocks = np.stack([np.stack([lists[(r * 2 + h) % len(lists)] for h in range(2)]) for r in range(s.rows.rows)])
    check_attention(s, q, 2, blocks)
    counts = (np.arange(s.rows.rows * 2, dtype=np.int32) % 4).reshape(-1, 2)
    check_attention(s, q, 2, blocks, counts)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kv", [17, 90, 1000, 5000])
def test_an_infinite_value_anywhere(dtype, kv):
    """A token of a generating sequence sees every key of its cache: the one infinite value comes out wherever it lies, and in
    its own component alone (rows of one share and of many)."""
    rng = np.random.default_rng(kv)
    s = Setup(rng, [1], [kv], 16, 1, 64, dtype, decode=True)
    q = normal(rng, (1, 4, 64), dtype)
    for key in sorted({0, 15, kv // 2, max(kv - 33, 0), max(kv - 17, 0), kv - 2, kv - 1}):
        at = int(s.table[0, key // 16]), 0, key % 16, key % 64
        was = s.v[at].clone()
        s.v[at] = float("-inf") if key % 2 else float("inf")
        check_attention(s, q, 1)
        s.v[at] = was


@pytest.mark.parametrize("low,high", [(0, 1 << 20), (1 << 27, 1 << 28), (1 << 30, (1 << 31) - 1), (-(1 << 31), -(1 << 30))])
def test_rotations_of_far_positions(low, high):
    """Unit vectors become cosine and sine of the fp64 angle. Those are within two fp32 steps, 2^-23, of exact for the fp32
    number next to the angle's fraction of a turn, and the correction for the rest is rounded once, 2^-25."""
    rng = np.random.default_rng(high % 1000)
    pos = rng.integers(low, high, 4096).astype(np.int32)
    pos[:2] = low, high - 1
    freq = np.concatenate([10000.0 ** (-np.arange(0, 32, 2) / 32), [0.999999, 1 / 3, 0.7, 1e-9]])
    x = torch.zeros((4096, 1, 40), device=DEV)
    x[:, :, :20] = 1.0
    y = A.spconv_rope(x, torch.from_numpy(pos).to(DEV), torch.from_numpy(freq).to(DEV))
    angle = pos.astype(np.float64)[:, None] * freq
    near(y[:, 0], np.concatenate([np.cos(angle), np.sin(angle)], 1), 2.0 ** -23 + 2.0 ** -25)


@pytest.mark.parametrize("keep", [0, 6])
def test_a_step_rotates_queries_and_keys_alike(keep):
    """Positions that the model counts from elsewhere than the sequence's first key: keys are stored as rotated by them, and
    the output is that of the scores between them."""
    rng = np.random.default_rng(71 + keep)
    dtype, heads, dim, block = torch.float32, 2, 64, 16
    layer = A.BlockAttention(30, heads, dim, block, keep, dtype=dtype, device=DEV)
    lens, B = [40, 23], 2
    s = Setup(rng, lens, lens, block, heads, dim, dtype, 8)
    q, k, v = (normal(rng, (s.tokens, h, dim), dtype) for h in (2 * heads, heads, heads))
    pos = np.concatenate([np.arange(n) * (b + 1) + 500 * b + 7 for b, n in enumerate(lens)]).astype(np.int32)
    dev_pos = torch.from_numpy(pos).to(DEV)
    out = layer.step(q, k, v, dev_pos, s.batch)
    freq = f64(layer.freq)
    want = O.rope(f64(k), pos, freq)
    bound = O.rope_bound(f64(k), freq, False, 1.0, dtype, want)
    for b in range(B):
        for i in range(lens[b]):
            t = int(s.start[b]) + i
            near(layer.k_cache[int(s.table[b, i // block]), :, i % block], want[t], bound[t], (b, i))
    rotated = layer.rotate(q, dev_pos)
    blocks, counts = layer.select(rotated, s.batch)
    host = lambda t: None if t is None else t.cpu().numpy()
    wo, _, bo, _ = O.attention(s.rows, f64(rotated), np.nan_to_num(f64(layer.k_cache)), np.nan_to_num(f64(layer.v_cache)), s.table, block,
                               dim ** -0.5, host(blocks), host(counts), dtype)
    near(out, wo, bo)


def test_a_rotation_of_what_requires_grad_is_refused():
    x = torch.randn((3, 2, 16), device=DEV, requires_grad=True)
    args = torch.arange(3, dtype=torch.int32, device=DEV), torch.ones(4, dtype=torch.float64, device=DEV)
    with pytest.raises(ValueError, match="requires grad"):
        A.spconv_rope(x, *args)
    with torch.no_grad():
        assert torch.equal(A.spconv_rope(x, *args), A.spconv_rope(x.detach(), *args))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("q_block", [1, 16])
def test_scores_of_sums_near_the_top_of_the_range(dtype, q_block):
    """Scores are products with the mean key: one that is finite comes out, also where that with the sum is not."""
    rng = np.random.default_rng(81 + q_block)
    s = Setup(rng, [20], [500], 64, 2, 64, dtype, q_block)
    sums = normal(rng, (s.pages, 2, 64), torch.float32)
    sums[int(s.table[0, 2])] *= 5e37
    sums[int(s.table[0, 4]), 1, 3] = 3.4e38
    sums[int(s.table[0, 7]), 0] *= 1e37  # a block of 52 keys
    q = normal(rng, (20, 8, 64), dtype)
    want, bound = O.scores(s.rows, f64(q), f64(sums), s.table, s.kv, 64, 2)
    assert np.abs(want[np.isfinite(want)]).max() < 2.0 ** 127
    near(A.spconv_block_scores(q, sums, s.batch), want, bound)
