"""GPU tests of the attention calls against their float64 forms (attention_oracle.py):
sizes, types, strides and masks where they can go wrong, streams, graphs, and the
calls of a step strung together. Tolerances are the oracle's bounds."""
import numpy as np
import pytest
import torch

import attention_oracle as O
from paper_2005_04091_amd import attention as A

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
DEV = "cuda:0"


def f64(t):
    return t.detach().double().cpu().numpy()


def normal(rng, shape, dtype, scale=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(DEV).to(dtype)


def near(got, want, bound, what=""):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        off = np.where(same, 0.0, np.abs(got - want))
    bad = ~(off <= bound) & ~same
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], want[bad][:4], np.broadcast_to(bound, got.shape)[bad][:4])


def strided(t, gap_token=0, gap_head=0):
    """The same values with other strides: gaps behind heads and tokens."""
    T, H, D = t.shape
    buf = torch.full((T, H * (D + gap_head) + gap_token), float("nan"), dtype=t.dtype, device=t.device)
    v = buf.as_strided((T, H, D), (buf.shape[1], D + gap_head, 1))
    v.copy_(t)
    return v


# ---- rotary positions ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H,D,rot,inter", [(1, 1, 2, 2, False), (5, 3, 128, 128, False), (7, 2, 104, 48, True), (3, 4, 81, 34, True),
                                             (3, 4, 81, 34, False), (1030, 2, 64, 32, False), (2, 1, 1024, 1024, True), (6, 5, 40, 0, False),
                                             (2049, 3, 96, 96, True)])
def test_rope(dtype, T, H, D, rot, inter):
    rng = np.random.default_rng(T * 31 + D)
    x = normal(rng, (T, H, D), dtype)
    pos = rng.integers(0, 1 << 20, T).astype(np.int32)
    pos[0] = 0x7fffffff if T > 1 else 0
    if T > 2:
        pos[1] = -5
    freq = 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    for inverse, amplitude in [(False, 1.0), (True, 1.25)]:
        want = O.rope(f64(x), pos, freq, inter, inverse, amplitude)
        bound = O.rope_bound(f64(x), freq, inter, amplitude, dtype, want)
        args = (torch.from_numpy(pos).to(DEV), torch.from_numpy(freq).to(DEV), inter, inverse, amplitude)
        got = A.spconv_rope(x, *args)
        near(got, want, bound)
        out = strided(torch.zeros_like(x), 3, 1)
        assert A.spconv_rope(strided(x, 5, 2), *args, out=out) is out
        near(out, want, bound, "strided")
        y = x.clone()
        A.spconv_rope(y, *args, out=y)
        assert torch.equal(y, got)
        assert torch.equal(A.spconv_rope(x[:, :1].expand(T, H, D), *args)[:, -1], got[:, 0])


@pytest.mark.parametrize("inter", [False, True])
def test_rope_gradient(inter):
    """The inverse is the gradient: against the formula's autograd, and against differences (the map is linear)."""
    rng = np.random.default_rng(8)
    T, H, D, rot, amp = 5, 2, 48, 32, 1.1
    freq = 10000.0 ** (-np.arange(0, rot, 2) / rot)
    pos = rng.integers(0, 5000, T).astype(np.int32)
    args = (torch.from_numpy(pos).to(DEV), torch.from_numpy(freq).to(DEV), inter)
    g = normal(rng, (T, H, D), torch.float32)
    x = torch.from_numpy(rng.standard_normal((T, H, D))).requires_grad_(True)
    angle = torch.from_numpy(pos.astype(np.float64)[:, None] * freq[None])
    c, s = (torch.cos(angle) * amp)[:, None], (torch.sin(angle) * amp)[:, None]
    i, j = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., i], x[..., j]
    ((a * c - b * s) * g.cpu()[..., i] + (b * c + a * s) * g.cpu()[..., j]).sum().add((x[..., rot:] * g.cpu()[..., rot:]).sum()).backward()
    got = A.spconv_rope(g, *args, inverse=True, amplitude=amp)
    near(got, x.grad.numpy(), O.rope_bound(f64(g), freq, inter, amp, torch.float32, x.grad.numpy()))
    # <g, R dx> = <R^T g, dx> for single components, up to the rounding of both sides.
    dx = torch.zeros(T, H, D, device=DEV)
    for d in (0, 1, rot // 2, rot - 1, D - 1):
        dx.zero_()
        dx[:, :, d] = 1.0
        left = f64(g * A.spconv_rope(dx, *args, amplitude=amp)).sum(-1)
        near(left, f64(got[:, :, d]), 8 * 2.0 ** -21 * np.abs(f64(g)).max())


# ---- batches ----

class Setup:
    """A random batch: sequences of `lens` tokens and `kv` keys, pages in random order with spare ones."""

    def __init__(self, rng, lens, kv, block, heads, dim, dtype, q_block=1, extra_cols=1, tail=0, decode=False):
        self.lens, self.kv, self.block = np.array(lens), np.array(kv), block
        B = len(lens)
        need = -(-self.kv // block)
        self.nb = int(max(need.max(), 1)) + extra_cols
        pages = int(need.sum()) + 4
        order = rng.permutation(pages)
        table = np.full((B, self.nb), -1, np.int32)
        at = 0
        for b in range(B):
            table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
        self.table, self.pages, self.spare = table, pages, order[at:]
        self.start = np.concatenate([[0], np.cumsum(self.lens)])
        self.tokens = int(self.start[-1]) + tail
        self.q_start = None if decode else self.start.astype(np.int32)
        self.rows = O.Rows(None if decode else self.start, self.kv, self.tokens, q_block)
        self.k = normal(rng, (pages, heads, block, dim), dtype)
        self.v = normal(rng, (pages, heads, block, dim), dtype)
        self.q_block = q_block
        self.make()

    def make(self):
        dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
        wide = np.full((self.table.shape[0], self.nb + 3), -7, np.int32)  # rows with a gap
        wide[:, :self.nb] = self.table
        self.batch = A.CacheBatch(dev(wide)[:, :self.nb], dev(self.kv.astype(np.int32)), self.block, dev(self.q_start), self.tokens,
                                  self.q_block)
        assert self.batch.rows == self.rows.rows


# ---- append ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,kv,block,heads,dim,rot,inter", [
    ([1], [1], 16, 1, 8, 8, False), ([1, 1, 1], [16, 17, 40], 16, 2, 64, 64, False), ([70, 0, 1, 33], [70, 5, 64, 200], 32, 3, 128, 64, True),
    ([5, 129], [300, 129], 128, 2, 256, 256, False), ([40], [55], 48, 2, 72, 20, True), ([9, 30], [9, 31], 256, 1, 96, 0, False)])
def test_append(dtype, lens, kv, block, heads, dim, rot, inter):
    rng = np.random.default_rng(dim + block)
    s = Setup(rng, lens, kv, block, heads, dim, dtype, tail=2)
    k, v = normal(rng, (s.tokens, heads, dim), dtype), normal(rng, (s.tokens, heads, dim), dtype)
    freq = 10000.0 ** (-np.arange(0, rot, 2) / rot) if rot else None
    for gap in (0, 1):
        kc, vc = s.k.clone(), s.v.clone()
        sums = torch.full((s.pages, heads, dim), 7.0, device=DEV)
        src = (strided(k, 3, gap), strided(v, 0, gap)) if gap else (k, v)
        A.spconv_cache_append(*src, kc, vc, s.batch, sums, None if freq is None else torch.from_numpy(freq).to(DEV), inter, 1.5)
        want_k, want_v, bound, touched = f64(s.k), f64(s.v), np.zeros(kc.shape), set()
        for b in range(len(lens)):
            for i in range(lens[b]):
                t, p = int(s.start[b]) + i, kv[b] - lens[b] + i
                page, slot = s.table[b, p // block], p % block
                x = f64(k[t:t + 1])
                y = x if freq is None else O.rope(x, np.array([p]), freq, inter, False, 1.5)
                want_k[page, :, slot], want_v[page, :, slot] = y[0], f64(v[t])
                bound[page, :, slot] = 0.0 if freq is None else O.rope_bound(x, freq, inter, 1.5, dtype, y)[0]
                touched.add((b, p // block))
        near(kc, want_k, bound, "keys")
        assert np.array_equal(f64(vc), want_v)
        got, stored = f64(sums), f64(kc)
        want = np.full(got.shape, 7.0)
        size = np.zeros(got.shape)
        for b, j in touched:
            page, n = s.table[b, j], min(block, kv[b] - j * block)
            want[page], size[page] = stored[page, :, :n].sum(1), np.abs(stored[page, :, :n]).sum(1)
        near(sums, want, size * block * O.U32, "sums")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,rot,inter", [(192, 192, True), (256, 168, False), (200, 0, False), (128, 26, True), (256, 2, False), (72, 64, False)])
def test_append_of_few_heads(dtype, dim, rot, inter):
    """Pages whose components several workgroups share: cache and sums against the formula, whole pages and part ones."""
    rng = np.random.default_rng(dim + rot)
    s = Setup(rng, [100, 3], [130, 40], 64, 1, dim, dtype, tail=1)
    k, v = (normal(rng, (s.tokens, 1, dim), dtype) for _ in range(2))
    freq = 500.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    kc, vc = s.k.clone(), s.v.clone()
    sums = torch.full((s.pages, 1, dim), 7.0, device=DEV)
    A.spconv_cache_append(k, v, kc, vc, s.batch, sums, torch.from_numpy(freq).to(DEV) if rot else None, inter)
    want_k, want_v = f64(s.k), f64(s.v)
    bound = np.zeros_like(want_k)
    touched = {}
    for b in range(2):
        n, kv, t0 = int(s.lens[b]), int(s.kv[b]), int(s.start[b])
        pos = np.arange(kv - n, kv).astype(np.int32)
        new = O.rope(f64(k)[t0:t0 + n], pos, freq, inter, False, 1.0)
        off = O.rope_bound(f64(k)[t0:t0 + n], freq, inter, 1.0, dtype, new)
        for i, p in enumerate(pos):
            page = int(s.table[b, p // 64])
            want_k[page, 0, p % 64], bound[page, 0, p % 64], want_v[page, 0, p % 64] = new[i, 0], off[i, 0], f64(v)[t0 + i, 0]
            touched[page] = min(kv - p // 64 * 64, 64)
    near(kc, want_k, bound)
    assert np.array_equal(f64(vc), want_v)
    for page in range(s.pages):
        if page not in touched:
            assert (sums[page] == 7.0).all()
            continue
        keys = f64(kc)[page, 0, :touched[page]]  # as stored: 64 fp32 additions at most
        near(sums[page, 0], keys.sum(0), np.abs(keys).sum(0) * 64 * 2.0 ** -24, page)


def test_append_again_after_dropped_tokens():
    """Drafted tokens that are dropped leave no trace in the sums."""
    rng = np.random.default_rng(3)
    s = Setup(rng, [12], [30], 16, 2, 64, torch.bfloat16)
    sums = torch.zeros((s.pages, 2, 64), device=DEV)
    k, v = normal(rng, (12, 2, 64), torch.bfloat16), normal(rng, (12, 2, 64), torch.bfloat16)
    A.spconv_cache_append(k, v, s.k, s.v, s.batch, sums)
    s.kv = np.array([27])  # the last four again, after one was dropped and nine kept
    s.start, s.q_start, s.tokens = np.array([0, 4]), np.array([0, 4], np.int32), 4
    s.rows = O.Rows(s.start, s.kv, 4, 1)
    s.make()
    A.spconv_cache_append(k[:4], v[:4], s.k, s.v, s.batch, sums)
    page = s.table[0, 1]
    near(sums[page], f64(s.k[page, :, :11]).sum(1), np.abs(f64(s.k[page, :, :11])).sum(1) * 16 * O.U32)


def test_append_drops_what_has_no_place():
    """Tokens before position 0, pages outside the cache: dropped; nothing else is touched."""
    rng = np.random.default_rng(4)
    s = Setup(rng, [20, 20, 3], [9, 40, 0], 16, 2, 64, torch.float16)
    s.table[1, 1], s.table[1, 2] = -1, s.pages
    s.make()
    kc, vc = s.k.clone(), s.v.clone()
    k, v = normal(rng, (43, 2, 64), torch.float16), normal(rng, (43, 2, 64), torch.float16)
    A.spconv_cache_append(k, v, kc, vc, s.batch)
    want_k, want_v = s.k.clone(), s.v.clone()
    page = int(s.table[0, 0])
    want_k[page, :, :9], want_v[page, :, :9] = k[11:20].transpose(0, 1), v[11:20].transpose(0, 1)
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)


# ---- scores ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,kv,block,heads,group,dim,q_block", [
    ([1], [1], 16, 1, 1, 8, 1), ([1, 1, 1], [100, 700, 16], 16, 2, 4, 128, 1), ([50, 0, 7], [300, 5, 7], 32, 2, 3, 64, 16),
    ([33, 64], [33, 200], 16, 1, 8, 256, 33), ([130], [1500], 16, 3, 5, 72, 128), ([9], [640], 64, 2, 20, 96, 1)])
def test_scores(dtype, lens, kv, block, heads, group, dim, q_block):
    rng = np.random.default_rng(dim + q_block)
    s = Setup(rng, lens, kv, block, heads, dim, dtype, q_block, extra_cols=3, tail=1)
    sums = normal(rng, (s.pages, heads, dim), torch.float32, 3.0)
    if s.table.shape[1] > 3:
        s.table[0, 1] = s.pages + 5  # not there
        s.make()
    q = normal(rng, (s.tokens, heads * group, dim), dtype)
    want, bound = O.scores(s.rows, f64(q), f64(sums), s.table, s.kv, block, heads)
    near(A.spconv_block_scores(q, sums, s.batch), want, bound)
    near(A.spconv_block_scores(strided(q, 1, 3), sums, s.batch), want, bound, "strided")


def test_scores_of_values_that_are_not_finite():
    rng = np.random.default_rng(6)
    s = Setup(rng, [20], [200], 16, 1, 64, torch.bfloat16, 16)
    sums = normal(rng, (s.pages, 1, 64), torch.float32)
    sums[s.table[0, 2], 0, 3] = float("inf")
    sums[s.table[0, 3], 0, 3] = float("nan")
    sums[s.table[0, 4], 0] = 3e38
    sums[s.table[0, 5], 0, :2] = torch.tensor([float("inf"), float("-inf")])
    q = normal(rng, (20, 4, 64), torch.bfloat16)
    q[:, :, :2] = q[:, :, :2].abs()
    q[7, 2, 5] = float("nan")
    q[9, 1, 5] = float("inf")
    want, bound = O.scores(s.rows, f64(q), f64(sums), s.table, s.kv, 16, 1)
    # fp32 products of 3e38 may pass the range where their exact sum does not.
    got = f64(A.spconv_block_scores(q, sums, s.batch))
    skip = [4]
    for j in range(s.nb):
        if j not in skip:
            near(got[:, :, j], want[:, :, j], bound[:, :, j], j)


# ---- selection ----

@pytest.mark.parametrize("nb,keep,sink,local,q_block,block", [
    (1, 1, 0, 1, 1, 16), (5, 3, 1, 1, 1, 16), (200, 16, 1, 2, 1, 16), (256, 17, 0, 0, 1, 16), (300, 40, 2, 3, 1, 16), (600, 7, 0, 2, 64, 32),
    (1100, 64, 1, 1, 1, 16), (2048, 100, 1, 2, 8, 16), (2049, 33, 1, 2, 1, 16), (5000, 1500, 3, 1, 1, 16), (70, 70, 1, 1, 1, 16),
    (33000, 50, 1, 1, 1, 16)])
def test_select(nb, keep, sink, local, q_block, block):
    rng = np.random.default_rng(nb)
    kv = [nb * block, max(1, nb * block - 7), max(1, nb * block // 3), 1]
    lens = [1, 1, 1, 1] if q_block == 1 else [min(q_block + 3, v) for v in kv]
    s = Setup(rng, lens, kv, block, 1, 8, torch.float32, q_block, extra_cols=0)
    H = 2
    sc = rng.standard_normal((s.rows.rows, H, nb)).astype(np.float32)
    sc[1 % s.rows.rows] = np.round(sc[1 % s.rows.rows] * 2) / 2  # many ties, of both zeros too
    sc[0, 0, rng.random(nb) < 0.3] = -0.0
    sc[0, 0, rng.random(nb) < 0.3] = 0.0
    sc[0, 1] = 1.5
    sc[min(2, s.rows.rows - 1)][:, rng.random(nb) < 0.9] = -np.inf
    sc[min(2, s.rows.rows - 1)][:, rng.random(nb) < 0.2] = np.nan
    sc[0, 0, rng.integers(0, nb)] = np.inf
    blocks, counts = A.spconv_select_blocks(torch.from_numpy(sc).to(DEV), s.batch, keep, sink, local)
    wb, wc = O.select(s.rows, sc, block, keep, sink, local)
    assert np.array_equal(counts.cpu().numpy(), wc)
    assert np.array_equal(blocks.cpu().numpy(), wb)


def test_select_reads_nothing_behind_the_visible_blocks():
    """Scores behind the visible blocks do not matter; rows without tokens get nothing; an empty cache neither."""
    rng = np.random.default_rng(12)
    s = Setup(rng, [5, 0, 9, 3], [100, 64, 40, 0], 16, 1, 8, torch.float32, 4, extra_cols=9)
    sc = torch.full((s.rows.rows, 1, s.nb), float("inf"), device=DEV)
    for r, (b, toks, pos) in s.rows.of.items():
        if pos[-1] >= 0:
            sc[r, :, :pos[-1] // 16 + 1] = torch.randn(pos[-1] // 16 + 1, device=DEV)
    blocks, counts = A.spconv_select_blocks(sc, s.batch, 3, 1, 1)
    wb, wc = O.select(s.rows, sc.cpu().numpy(), 16, 3, 1, 1)
    assert np.array_equal(blocks.cpu().numpy(), wb) and np.array_equal(counts.cpu().numpy(), wc)


# ---- attention ----

def random_lists(rng, s, heads, keep):
    """Lists with repeats, entries out of range and blocks behind the row's tokens; counts of all kinds."""
    blocks = rng.integers(-1, s.nb + 1, (s.rows.rows, heads, keep)).astype(np.int32)
    counts = rng.integers(0, keep + 3, (s.rows.rows, heads)).astype(np.int32)
    counts[rng.random(counts.shape) < 0.1] = -2
    return blocks, counts


def check_attention(s, q, heads, blocks=None, counts=None, scale=None, k=None, v=None):
    dev = lambda a: None if a is None else torch.from_numpy(a).to(DEV)
    D = q.shape[2]
    out = torch.full(q.shape, 3.0, dtype=q.dtype, device=DEV)
    lse = torch.full(q.shape[:2], 3.0, device=DEV)
    k, v = s.k if k is None else k, s.v if v is None else v
    A.spconv_block_attention(q, k, v, s.batch, dev(blocks), dev(counts), scale, out, lse)
    wo, wl, bo, bl = O.attention(s.rows, f64(q), f64(k), f64(v), s.table, s.block, D ** -0.5 if scale is None else scale, blocks, counts,
                                 q.dtype)
    mine = np.zeros(q.shape[0], bool)
    for _, toks, _ in s.rows.of.values():
        mine[toks] = True
    near(f64(out)[mine], wo[mine], bo[mine], "out")
    near(f64(lse)[mine], wl[mine], bl[mine], "lse")
    assert (f64(out)[~mine] == 3.0).all() and (f64(lse)[~mine] == 3.0).all()
    return out, lse


CASES = [
    # lens, kv, block, heads, group, dim, q_block, decode
    ([1], [1], 16, 1, 1, 8, 1, True), ([1, 1, 1], [5, 100, 333], 16, 2, 4, 128, 1, True), ([1], [3000], 64, 2, 8, 128, 1, True),
    ([1, 1], [700, 90], 48, 1, 20, 80, 1, True), ([50, 0, 7], [300, 5, 7], 32, 2, 3, 64, 16, False),
    ([33, 64], [33, 200], 16, 1, 8, 256, 33, False), ([130], [500], 128, 2, 4, 128, 64, False), ([90, 5], [90, 260], 64, 1, 5, 96, 128, False),
    ([17], [40], 16, 3, 1, 72, 1, False), ([4, 4], [1000, 100], 256, 1, 16, 192, 4, False), ([257], [257], 32, 1, 2, 64, 128, False),
    ([3], [2], 16, 1, 2, 64, 2, False)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES, ids=str)
def test_attention(dtype, case):
    lens, kv, block, heads, group, dim, q_block, decode = case
    rng = np.random.default_rng(sum(kv) + dim)
    s = Setup(rng, lens, kv, block, heads, dim, dtype, q_block, extra_cols=2, tail=0 if decode else 3, decode=decode)
    q = normal(rng, (s.tokens, heads * group, dim), dtype)
    check_attention(s, q, heads)
    blocks, counts = random_lists(rng, s, heads, 7)
    check_attention(s, strided(q, 3, 1), heads, blocks, counts)
    check_attention(s, strided(q, 16, 8), heads, blocks, None, scale=-0.2)
    if s.nb > 2:
        s.table[0, 1] = -1
        s.make()
        check_attention(s, q, heads)


WIDE = [
    # lens, kv, block, heads, group, dim, q_block: wide heads in rows and in tiles of 64 and 128 pairs; lists longer than one
    # look-up; more (row, head) items than the GPU holds at a time, with a rest that is split along its keys
    ([5], [300], 32, 1, 2, 160, 1), ([20, 3], [150, 3], 16, 2, 4, 192, 8), ([70], [600], 64, 1, 4, 200, 33), ([40], [90], 16, 1, 8, 256, 16),
    ([3, 9], [5000, 4500], 256, 1, 2, 32, 4), ([66], [4800], 128, 1, 4, 40, 64), ([530], [700], 16, 1, 2, 24, 1), ([4200], [4210], 256, 2, 2, 16, 16),
    ([3], [4700], 64, 1, 1, 256, 1)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", WIDE, ids=str)
def test_attention_wide_long_and_many(dtype, case):
    lens, kv, block, heads, group, dim, q_block = case
    rng = np.random.default_rng(sum(kv) * 3 + dim)
    s = Setup(rng, lens, kv, block, heads, dim, dtype, q_block, extra_cols=1, tail=2)
    q = normal(rng, (s.tokens, heads * group, dim), dtype)
    check_attention(s, q, heads)
    blocks, counts = random_lists(rng, s, heads, max(5, 4400 // block if kv[0] > 4400 else 5))
    check_attention(s, q, heads, blocks, counts)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("q_block,group", [(1, 2), (8, 4), (64, 4)])
def test_attention_of_a_scale_of_zero(dtype, q_block, group):
    """Every seen key weighs the same, also where the keys are split and joined."""
    rng = np.random.default_rng(q_block + 40)
    s = Setup(rng, [9], [900], 16, 1, 64, dtype, q_block)
    q = normal(rng, (s.tokens, group, 64), dtype)
    blocks, counts = random_lists(rng, s, 1, 50)
    check_attention(s, q, 1, blocks, counts, scale=0.0)
    check_attention(s, q, 1, scale=0.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,q_block", [(192, 1), (256, 1), (200, 16), (256, 16)])
def test_attention_of_wide_values_that_are_not_finite(dtype, dim, q_block):
    rng = np.random.default_rng(dim + q_block)
    s = Setup(rng, [21], [90], 16, 1, dim, dtype, q_block)
    q = normal(rng, (s.tokens, 4, dim), dtype)
    for pos, d, x in [(80, 3, "inf"), (84, dim - 1, "nan"), (84, 5, "-inf"), (89, 7, "inf"), (10, 9, "inf"), (83, 100, "-inf"), (85, 100, "inf")]:
        s.v[int(s.table[0, pos // 16]), 0, pos % 16, d] = float(x)
    check_attention(s, q, 1)
    blocks, counts = random_lists(rng, s, 1, 6)
    check_attention(s, q, 1, blocks, counts)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("q_block,group", [(1, 4), (16, 2), (64, 4)])
def test_attention_what_is_masked_takes_no_part(dtype, q_block, group):
    """NaN and infinities in slots behind the newest key, in keys and values that a part of the row's tokens does not see
    yet, and in pages that nobody lists."""
    rng = np.random.default_rng(q_block)
    n = 1 if q_block == 1 else 70
    s = Setup(rng, [n, n], [75, 150], 32, 2, 64, dtype, q_block)
    bad = [float("nan"), float("inf"), float("-inf")]
    for b in range(2):
        kv = s.kv[b]
        page = int(s.table[b, (kv - 1) // 32])
        for t in (s.k, s.v):
            t[page, :, (kv - 1) % 32 + 1:] = bad[0]
    for p in s.spare:
        s.k[p], s.v[p] = bad[0], bad[0]
    q = normal(rng, (s.tokens, 2 * group, 64), dtype)
    check_attention(s, q, 2)
    if n > 1:
        # Seen by the last tokens alone: theirs are not finite, the others' stay as they are.
        for b in range(2):
            j = int(s.kv[b]) - 9
            page, slot = int(s.table[b, j // 32]), j % 32
            s.v[page, :, slot, 5] = bad[1]
            s.v[page, :, slot, 40] = bad[0]
            s.v[page, 1, (slot + 1) % 32, 6] = bad[2]
        check_attention(s, q, 2)
        for b in range(2):
            j = int(s.kv[b]) - 4
            s.k[int(s.table[b, j // 32]), 0, j % 32, 3] = bad[0]
        check_attention(s, q, 2)


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_extreme_scores(dtype):
    """Scores of hundreds (weights that vanish), equal ones, and a query of zeros."""
    rng = np.random.default_rng(5)
    s = Setup(rng, [40, 1], [90, 400], 16, 1, 64, dtype, 32)
    q = normal(rng, (s.tokens, 4, 64), dtype, 30.0)
    q[3] = 0
    check_attention(s, q, 1)
    s.k[int(s.table[0, 0]), 0, :] = s.k[int(s.table[0, 0]), 0, :1].clone()
    check_attention(s, q, 1)


def test_attention_is_reproducible_and_in_place_of_splits():
    """Same bits run to run, on another stream, and with a workspace that holds garbage."""
    rng = np.random.default_rng(9)
    s = Setup(rng, [1, 1], [4000, 77], 64, 2, 128, torch.bfloat16, decode=True)
    q = normal(rng, (2, 8, 128), torch.bfloat16)
    first = A.spconv_block_attention(q, s.k, s.v, s.batch, lse=True)
    n = A.spconv_attention_workspace(torch.bfloat16, s.batch, 8, 2, 128)
    assert n > 0
    ws = torch.full((n + 16,), 255, dtype=torch.uint8, device=DEV)
    again = A.spconv_block_attention(q, s.k, s.v, s.batch, lse=True, workspace=ws[:n])
    assert all(torch.equal(a, b) for a, b in zip(first, again)) and (ws[n:] == 255).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    third = A.spconv_block_attention(q, s.k, s.v, s.batch, lse=True, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, third))
    with pytest.raises(A.SpconvError):
        A.spconv_block_attention(q, s.k, s.v, s.batch, workspace=ws[:n - 16])


def test_offsets_past_32_bits():
    """A cache of more than 2^32 elements: pages at its end, table entries that are large."""
    pages, heads, block, dim = 33000, 8, 128, 128  # 4.3e9 elements, 8.7 GB each
    k = torch.zeros((pages, heads, block, dim), dtype=torch.float16, device=DEV)
    v = torch.zeros_like(k)
    rng = np.random.default_rng(2)
    table = np.array([[32999, 5, 32768, 31000]], np.int32)
    batch = A.CacheBatch(torch.from_numpy(table).to(DEV), torch.tensor([450], dtype=torch.int32, device=DEV), 128,
                         torch.tensor([0, 450], dtype=torch.int32, device=DEV), 450, 64)
    kn, vn = normal(rng, (450, heads, dim), torch.float16), normal(rng, (450, heads, dim), torch.float16)
    sums = torch.zeros((pages, heads, dim), device=DEV)
    A.spconv_cache_append(kn, vn, k, v, batch, sums)
    for j in range(4):
        n = min(128, 450 - j * 128)
        assert torch.equal(k[table[0, j], :, :n], kn[j * 128:j * 128 + n].transpose(0, 1))
        assert torch.equal(v[table[0, j], :, :n], vn[j * 128:j * 128 + n].transpose(0, 1))
    assert int((sums != 0).any(2).any(1).sum()) == 4
    q = normal(rng, (450, 8, dim), torch.float16)
    got = A.spconv_block_attention(q, k, v, batch)
    # The same on a small cache.
    small = torch.from_numpy(np.arange(4, dtype=np.int32)[None]).to(DEV)
    at = torch.from_numpy(table[0].astype(np.int64)).to(DEV)
    b2 = A.CacheBatch(small, batch.kv_len, 128, batch.q_start, 450, 64)
    assert torch.equal(got, A.spconv_block_attention(q, k[at].contiguous(), v[at].contiguous(), b2))
    s2 = A.spconv_block_scores(q, sums, batch)
    assert torch.equal(s2, A.spconv_block_scores(q, sums[at].contiguous(), b2))


# ---- the calls of a step together ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("keep", [0, 5])
def test_a_prompt_then_single_tokens(dtype, keep):
    """A prompt in two parts, then single tokens, through BlockAttention: every step's output against attention in float64
    over the cache as it is stored, with the lists that a float64 selection would accept."""
    rng = np.random.default_rng(21)
    heads, group, dim, block, B = 2, 3, 64, 16, 2
    layer = A.BlockAttention(40, heads, dim, block, keep, 1, 2, rot=32, dtype=dtype, device=DEV,
                             scaling=dict(kind="by_parts", factor=4.0, low=1.0, high=4.0, original=64.0))
    order = rng.permutation(40)
    table = order.reshape(B, 20).astype(np.int32)
    tab = torch.from_numpy(table).to(DEV)
    kv = np.zeros(B, np.int64)
    freq = f64(layer.freq)
    for step, lens in enumerate([[70, 33], [40, 64], [1, 1], [1, 1]]):
        n, qb = np.array(lens), 1 if max(lens) == 1 else 32
        kv = kv + n
        start = np.concatenate([[0], np.cumsum(n)])
        T = int(start[-1])
        rows = O.Rows(start, kv, T, qb)
        batch = A.CacheBatch(tab, torch.from_numpy(kv.astype(np.int32)).to(DEV), block,
                             None if qb == 1 else torch.from_numpy(start.astype(np.int32)).to(DEV), T, qb)
        q, k, v = normal(rng, (T, heads * group, dim), dtype), normal(rng, (T, heads, dim), dtype), normal(rng, (T, heads, dim), dtype)
        pos = np.concatenate([np.arange(kv[b] - n[b], kv[b]) for b in range(B)]).astype(np.int32)
        out, lse = layer.step(q, k, v, torch.from_numpy(pos).to(DEV), batch, lse=True)
        rotated = layer.rotate(q, torch.from_numpy(pos).to(DEV))
        want_q = O.rope(f64(q), pos, freq)
        near(rotated, want_q, O.rope_bound(f64(q), freq, False, 1.0, dtype, want_q))
        blocks, counts = layer.select(rotated, batch)
        if keep:
            exact, bound = O.scores(rows, f64(rotated), f64(layer.sums), table, kv, block, heads)
            got = blocks.cpu().numpy()
            for r, (b, toks, p) in rows.of.items():
                n_vis = p[-1] // block + 1
                low = p[0] // block - 1
                for h in range(heads):
                    chosen = set(got[r, h][:int(counts[r, h])].tolist())
                    assert len(chosen) == min(keep, n_vis)
                    if n_vis > keep:
                        assert 0 in chosen and set(range(max(low, 0), n_vis)) <= chosen
                        free = [j for j in chosen if 1 <= j < low]
                        rest = [j for j in range(1, max(low, 1)) if j not in chosen]
                        for i in free:
                            for j in rest:
                                assert exact[r, h, i] + bound[r, h, i] >= exact[r, h, j] - bound[r, h, j]
            # The sums are those of the stored keys.
            for b in range(B):
                for j in range(-(-int(kv[b]) // block)):
                    keys = f64(layer.k_cache[int(table[b, j]), :, :min(block, int(kv[b]) - j * block)])
                    near(layer.sums[int(table[b, j])], keys.sum(1), np.abs(keys).sum(1) * block * O.U32)
        wo, wl, bo, bl = O.attention(rows, f64(rotated), np.nan_to_num(f64(layer.k_cache)), np.nan_to_num(f64(layer.v_cache)), table, block,
                                     dim ** -0.5, blocks.cpu().numpy() if keep else None, counts.cpu().numpy() if keep else None, dtype)
        near(out, wo, bo, step)
        near(lse, wl, bl, step)


def test_a_step_in_a_graph():
    """A captured step, replayed with other inputs and lengths in the same buffers, with eager work between the replays."""
    rng = np.random.default_rng(30)
    heads, dim, block, B = 2, 128, 32, 3
    layer = A.BlockAttention(120, heads, dim, block, 6, 1, 2, dtype=torch.bfloat16, device=DEV)
    layer.k_cache.normal_()
    layer.v_cache.normal_()
    layer.sums.normal_()
    table = torch.from_numpy(rng.permutation(120).reshape(B, 40).astype(np.int32)).to(DEV)
    kv = torch.tensor([1000, 1, 517], dtype=torch.int32, device=DEV)
    pos = torch.zeros(B, dtype=torch.int32, device=DEV)
    q = torch.zeros((B, 8, dim), dtype=torch.bfloat16, device=DEV)
    k, v = (torch.zeros((B, heads, dim), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    batch = A.CacheBatch(table, kv, block)

    def load(i):
        r = np.random.default_rng(100 + i)
        for t in (q, k, v):
            t.copy_(normal(r, tuple(t.shape), torch.bfloat16))
        kv.copy_(torch.from_numpy(r.integers(1, 1280, B).astype(np.int32)))
        pos.copy_(kv - 1)

    load(0)
    state = [t.clone() for t in (layer.k_cache, layer.v_cache, layer.sums)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.step(q, k, v, pos, batch, lse=True)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = layer.step(q, k, v, pos, batch, lse=True)
    for i in range(4):
        load(i)
        for t, c in zip((layer.k_cache, layer.v_cache, layer.sums), state):
            t.copy_(c)
        eager = [t.clone() for t in layer.step(q, k, v, pos, batch, lse=True)]
        after = [t.clone() for t in (layer.k_cache, layer.v_cache, layer.sums)]
        for t, c in zip((layer.k_cache, layer.v_cache, layer.sums), state):
            t.copy_(c)
        for t in held:
            t.fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(held, eager)), i
        assert all(torch.equal(a, b) for a, b in zip((layer.k_cache, layer.v_cache, layer.sums), after)), i


@pytest.mark.parametrize("B,q_block", [(70, 1), (70, 4), (5000, 1), (5000, 8)])
def test_many_short_sequences(B, q_block):
    """Rows are found among more sequences than a wave compares at a time, empty ones among them."""
    rng = np.random.default_rng(B + q_block)
    lens = rng.integers(0, 3, B) if B > 100 else rng.integers(0, 12, B)
    s = Setup(rng, lens, lens + rng.integers(0, 20, B), 16, 1, 16, torch.bfloat16, q_block, tail=1)
    q = normal(rng, (s.tokens, 2, 16), torch.bfloat16)
    check_attention(s, q, 1)
    blocks, counts = random_lists(rng, s, 1, 3)
    check_attention(s, q, 1, blocks, counts)
    sums = torch.randn((s.pages, 1, 16), device=DEV)
    want, bound = O.scores(s.rows, f64(q), f64(sums), s.table, s.kv, 16, 1)
    got = A.spconv_block_scores(q, sums, s.batch)
    near(got, want, bound)
    wb, wc = O.select(s.rows, got.cpu().numpy(), 16, 2, 0, 1)
    blocks, counts = A.spconv_select_blocks(got, s.batch, 2, 0, 1)
    assert np.array_equal(blocks.cpu().numpy(), wb) and np.array_equal(counts.cpu().numpy(), wc)
    # Keys of every sequence end up at the end of its pages.
    k, v = (normal(rng, (s.tokens, 1, 16), torch.bfloat16) for _ in range(2))
    kc, vc = s.k.clone(), s.v.clone()
    A.spconv_cache_append(k, v, kc, vc, s.batch)
    for b in range(0, B, 1 if B < 100 else 37):
        for i in range(lens[b]):
            at = s.kv[b] - lens[b] + i
            page = int(s.table[b, at // 16])
            assert torch.equal(kc[page, 0, at % 16], k[s.start[b] + i, 0]) and torch.equal(vc[page, 0, at % 16], v[s.start[b] + i, 0])


def test_sequences_that_share_their_first_pages():
    rng = np.random.default_rng(51)
    for q_block, lens in ((1, [3, 2, 5]), (8, [20, 9, 33])):
        s = Setup(rng, lens, [200, 180, 222], 16, 2, 64, torch.float16, q_block)
        s.table[1, :9] = s.table[2, :9] = s.table[0, :9]
        s.make()
        q = normal(rng, (s.tokens, 6, 64), torch.float16)
        k, v = (normal(rng, (s.tokens, 2, 64), torch.float16) for _ in range(2))
        sums = torch.randn((s.pages, 2, 64), device=DEV)
        before = sums.clone()
        A.spconv_cache_append(k, v, s.k, s.v, s.batch, sums)
        shared = torch.from_numpy(s.table[0, :9].astype(np.int64)).to(DEV)
        assert torch.equal(sums[shared], before[shared])  # only read
        want, bound = O.scores(s.rows, f64(q), f64(sums), s.table, s.kv, 16, 2)
        scores = A.spconv_block_scores(q, sums, s.batch)
        near(scores, want, bound)
        blocks, counts = A.spconv_select_blocks(scores, s.batch, 8, 1, 2)
        check_attention(s, q, 2, blocks.cpu().numpy(), counts.cpu().numpy())
        check_attention(s, q, 2)


@pytest.mark.parametrize("keep,q_block", [(6, 16), (0, 16), (5, 1)])
def test_prompts_in_a_graph(keep, q_block):
    """A captured step of ragged prompts, replayed after others of other lengths in the same buffers."""
    rng = np.random.default_rng(keep + q_block)
    heads, dim, block, B, T = 2, 64, 16, 3, 90
    layer = A.BlockAttention(130, heads, dim, block, keep, 1, 2, dtype=torch.float16, device=DEV)
    layer.k_cache.normal_()
    layer.v_cache.normal_()
    if keep:
        layer.sums.normal_()
    state = [t.clone() for t in (layer.k_cache, layer.v_cache, layer.sums) if t is not None]
    table = torch.from_numpy(rng.permutation(130)[:120].reshape(B, 40).astype(np.int32)).to(DEV)
    kv = torch.zeros(B, dtype=torch.int32, device=DEV)
    start = torch.zeros(B + 1, dtype=torch.int32, device=DEV)
    pos = torch.zeros(T, dtype=torch.int32, device=DEV)
    q = torch.zeros((T, 4, dim), dtype=torch.float16, device=DEV)
    k, v = (torch.zeros((T, heads, dim), dtype=torch.float16, device=DEV) for _ in range(2))
    batch = A.CacheBatch(table, kv, block, start, T, q_block)
    out, lse = torch.zeros_like(q), torch.zeros((T, 4), device=DEV)

    def load(i):
        r = np.random.default_rng(200 + i)
        for t in (q, k, v):
            t.copy_(normal(r, tuple(t.shape), torch.float16))
        cut = np.sort(r.integers(0, T + 1, B + 1)).astype(np.int32)
        lens = np.diff(cut)
        keys = (lens + r.integers(0, 640 - T, B)).astype(np.int32)
        start.copy_(torch.from_numpy(cut))
        kv.copy_(torch.from_numpy(keys))
        p = np.zeros(T, np.int32)
        for b in range(B):
            p[cut[b]:cut[b + 1]] = np.arange(keys[b] - lens[b], keys[b])
        pos.copy_(torch.from_numpy(p))

    def fresh():
        for t, c in zip([t for t in (layer.k_cache, layer.v_cache, layer.sums) if t is not None], state):
            t.copy_(c)
        out.fill_(5.0)
        lse.fill_(5.0)

    load(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.step(q, k, v, pos, batch, out, lse)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(q, k, v, pos, batch, out, lse)
    for i in range(4):
        load(i)
        fresh()
        layer.step(q, k, v, pos, batch, out, lse)
        eager = [out.clone(), lse.clone(), layer.k_cache.clone()]
        fresh()
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip((out, lse, layer.k_cache), eager)), i


def test_a_stream_of_another_device_is_refused():
    class Elsewhere:
        device, cuda_stream = torch.device("cuda", 7), 0

    x = torch.zeros((1, 1, 8), device=DEV)
    with pytest.raises(ValueError):
        A.spconv_rope(x, torch.zeros(1, dtype=torch.int32, device=DEV), torch.ones(2, dtype=torch.float64, device=DEV), stream=Elsewhere())


def test_queries_as_outputs_are_refused():
    s = Setup(np.random.default_rng(1), [1], [20], 16, 1, 8, torch.float32, decode=True)
    q = torch.zeros((1, 1, 8), device=DEV)
    with pytest.raises(A.SpconvError):
        A.spconv_block_attention(q, s.k, s.v, s.batch, out=q)


def test_two_streams_at_once():
    """Two steps on two streams with workspaces of their own give their serial results."""
    rng = np.random.default_rng(33)
    work = []
    for i in range(2):
        s = Setup(rng, [1] * 4, [900 + 300 * i, 10, 444, 77], 32, 2, 64, torch.float16, decode=True)
        work.append((s, normal(rng, (4, 8, 64), torch.float16)))
    serial = [A.spconv_block_attention(q, s.k, s.v, s.batch, lse=True) for s, q in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    got = [[] for _ in work]
    for _ in range(5):
        for i, (s, q) in enumerate(work):
            got[i].append(A.spconv_block_attention(q, s.k, s.v, s.batch, lse=True, stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for o, l in got[i]:
            assert torch.equal(o, serial[i][0]) and torch.equal(l, serial[i][1])


def test_malformed_sequences_stay_in_bounds():
    """Starts that decrease, lie outside the tokens or leave some out, and lengths out of range: whatever comes out, tokens
    that no sequence has are left as they are, and nothing outside the buffers is touched (guards around the outputs)."""
    rng = np.random.default_rng(40)
    s = Setup(rng, [6, 6, 6], [60, 40, 50], 16, 1, 64, torch.bfloat16, 4)
    q = normal(rng, (18, 2, 64), torch.bfloat16)
    for starts, kv in [([3, 9, 4, 18], [60, 40, 50]), ([-5, 6, 12, 400], [60, 40, 50]), ([18, 12, 6, 0], [60, 40, 50]),
                       ([0, 6, 12, 18], [-3, 100000, 50]), ([7, 7, 7, 7], [60, 40, 50])]:
        for qb in (1, 4):
            batch = A.CacheBatch(s.batch.table, torch.tensor(kv, dtype=torch.int32, device=DEV), 16,
                                 torch.tensor(starts, dtype=torch.int32, device=DEV), 18, qb)
            guard = torch.full((18 + 2, 2, 64), 3.0, dtype=torch.bfloat16, device=DEV)
            A.spconv_block_attention(q, s.k, s.v, batch, out=guard[1:-1])
            assert (guard[0] == 3.0).all() and (guard[-1] == 3.0).all()
            if starts == [7, 7, 7, 7]:
                assert (guard == 3.0).all()
            sc = A.spconv_block_scores(q, torch.zeros((s.pages, 1, 64), device=DEV), batch)
            blocks, counts = A.spconv_select_blocks(sc, batch, 4)
            assert int(blocks.min()) >= -1 and int(blocks.max()) < s.nb and int(counts.max()) <= 4
            kc, vc = s.k.clone(), s.v.clone()
            A.spconv_cache_append(q[:, :1], q[:, 1:], kc, vc, batch)
    torch.cuda.synchronize()
