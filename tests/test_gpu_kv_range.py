"""Attention over the paged 8-bit cache at the ends of the range: scores and values as large or as small as 16-bit inputs make them, in both kernels.  The content is read
back by gather, and rows are compared with 64 bits over the keys that they see; what a row does not see must not matter to it."""
import numpy as np
import pytest

from paper_2411_05007_amd import svdq as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# new tokens of a sequence and how often the batch holds it: single tokens (the kernel of few rows), and so many rows that the kernel of many takes them
FEW, MANY = (1, 1), (200, 256)


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "these tests need the MI355X"
    S.lib()
    return t


@pytest.fixture(scope="module")
def KV(torch):
    from paper_2411_05007_amd import kv
    return kv


class Sequence:
    """Keys and values fp32 [L, heads, D] in a cache, and what it holds of them in 64 bits."""

    def __init__(self, torch, KV, k, v, page=64):
        self.torch, self.KV = torch, KV
        self.L, self.heads, self.D = k.shape
        pages = (self.L + page - 1) // page
        self.cache = KV.KVCache(pages, self.heads, self.D, page)
        self.table = torch.arange(pages, dtype=torch.int32, device=DEV)[None].contiguous()
        self.cache.append(k.to(DEV).to(torch.bfloat16), v.to(DEV).to(torch.bfloat16), KV.KVBatch(self.i32([0, self.L]), self.i32([self.L]), self.table, self.L, self.L, self.L))
        self.k, self.v = (t.double().cpu() for t in self.cache.gather(KV.KVRows(self.i32([0]), self.i32([0, self.L]), self.table, self.L)))

    def i32(self, x):
        return self.torch.tensor(np.asarray(x), dtype=self.torch.int32, device=DEV)

    def attend(self, q, copies=1, length=None, max_new=None, **kw):
        """q fp32 [new, q_heads, D], the sequence's last tokens, in a batch that holds it `copies` times; fp64 [new, q_heads, D]"""
        torch, new, length = self.torch, q.shape[0], self.L if length is None else length
        q = q.to(DEV).to(torch.bfloat16)
        batch = self.KV.KVBatch(self.i32(np.arange(copies + 1) * new), self.i32([length] * copies), self.table.expand(copies, -1).contiguous(), new * copies,
                                new if max_new is None else max_new, length)
        out = torch.full((new * copies, q.shape[1], self.D), 7.0, dtype=torch.bfloat16, device=DEV)
        out = self.cache.attention(q.repeat(copies, 1, 1), batch, out=out, **kw).view(copies, *q.shape)
        assert torch.equal(out[0].view(torch.int16), out[copies - 1].view(torch.int16))
        return out[copies // 2].double().cpu(), q.double().cpu()

    def seen(self, i, new, causal=True, window=0):
        pos = self.L - new + i
        return slice(max(0, pos + 1 - window) if causal and window else 0, pos + 1 if causal else self.L)

    def want(self, q, i, h, causal=True, window=0, scale=None):
        """row i and head h of the output, and the weighted sum of magnitudes"""
        keys, kh = self.seen(i, q.shape[0], causal, window), h // (q.shape[1] // self.heads)
        p = self.torch.softmax(self.k[keys, kh] @ q[i, h] * (self.D ** -0.5 if scale is None else scale), 0)
        return p @ self.v[keys, kh], p @ self.v[keys, kh].abs()


def normal(torch, seed, *shape):
    gen = torch.Generator()
    gen.manual_seed(seed)
    return torch.randn(*shape, generator=gen)


@pytest.mark.parametrize("new,copies", [FEW, MANY])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_scores_near_the_lowest_number_are_scores(torch, KV, dim, new, copies):
    """Every key the same, every score -2^100 sqrt(dim) (of powers of two, so that they are exact): the mean of the values."""
    w = Sequence(torch, KV, torch.full((300, 1, dim), 2.0 ** 50), normal(torch, dim, 300, 1, dim))
    got, _ = w.attend(torch.full((new, 2, dim), -2.0 ** 50), copies)
    for i in {0, new - 1}:
        v = w.v[w.seen(i, new), 0]
        # equal weights are exact; fp32 sums of 300 products, a bf16 output
        assert ((got[i] - v.mean(0)).abs() <= 2.0 ** -8 * v.mean(0).abs() + 2.0 ** -14 * v.abs().mean(0)).all()


@pytest.mark.parametrize("new,copies", [FEW, MANY, (300, 1)])
@pytest.mark.parametrize("dim,size", [(64, 2.0 ** 12), (64, 2.0 ** 16), (128, 2.0 ** 14), (128, 2.0 ** 21), (128, 2.0 ** 40), (256, 2.0 ** 17)])
def test_scores_of_any_size_have_a_largest(torch, KV, dim, size, new, copies):
    """Scores of about 16 size^2.  Queries without a rotation are exact in f16 and codes are exact, so a score is off by the fp32 sum of its products alone, 2^-16 of their
    magnitudes: where the second largest is farther than that and 40 below the largest, the row is the value of its largest key, rounded to 16 bits."""
    L = 9000 if new == 300 else 300      # (300 rows on so many keys: in parts)
    w = Sequence(torch, KV, normal(torch, 1, L, 1, dim) * size, normal(torch, 2, L, 1, dim))
    got, q = w.attend(normal(torch, 3, new, 2, dim) * size, copies)
    checked = 0
    for i in {0, 1, new // 2, new - 1} & set(range(new)):
        for h in range(2):
            keys = w.k[w.seen(i, new), 0]
            score = keys @ q[i, h] * dim ** -0.5
            top = score.topk(2)
            off = 2.0 ** -16 * (keys.abs() @ q[i, h].abs()).max() * dim ** -0.5
            if top.values[0] - top.values[1] > 40 + 2 * off:
                want = w.v[top.indices[0], 0]
                assert ((got[i, h] - want).abs() <= 2.0 ** -8 * want.abs()).all(), (i, h)
                checked += 1
    assert checked > 0


@pytest.mark.parametrize("new,copies", [FEW, MANY])
@pytest.mark.parametrize("size", [2.0 ** 9, 2.0 ** 13, 2.0 ** 15, 2.0 ** 16, 2.0 ** 25])
def test_equal_scores_of_any_size_weigh_the_same(torch, KV, size, new, copies):
    """Two equal keys above all others, whatever their score is rounded to: the mean of their values."""
    k, q = normal(torch, 4, 300, 1, 128), normal(torch, 5, 1, 1, 128)
    k[70] = k[71] = q[0] * 4
    w = Sequence(torch, KV, k * size, normal(torch, 6, 300, 1, 128))
    got, _ = w.attend((q * size).expand(new, 2, 128), copies)
    want = w.v[70:72, 0].mean(0)
    assert ((got[[0, new - 1]] - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -16 * w.v[70:72, 0].abs().sum(0)).all()


@pytest.mark.parametrize("new,copies", [FEW, MANY])
def test_a_score_that_passes_fp32_is_not_left_out(torch, KV, new, copies):
    """q and k finite, their product not: NaN, not the answer without that key."""
    k, v = normal(torch, 7, 300, 1, 64), normal(torch, 8, 300, 1, 64)
    k[50] = 1e25
    w = Sequence(torch, KV, k, v)
    got, _ = w.attend(torch.full((new, 1, 64), 1e25), copies)
    assert bool(torch.isnan(got[[0, new - 1]]).all())


def close(w, got, q, i, h, **kw):
    """Row i and head h within what its arithmetic allows: queries without a rotation are exact in f16, fp32 scores are off by 2^-16 of their products' magnitudes, weights are
    rounded to 11 bits and summed in fp32, the output to 8; what is below 2^-33 of the largest weight may be left out, of the values that the row sees."""
    want, size = w.want(q, i, h, **kw)
    keys, kh = w.seen(i, q.shape[0], kw.get("causal", True), kw.get("window", 0)), h // (q.shape[1] // w.heads)
    scale = w.D ** -0.5 if kw.get("scale") is None else abs(kw["scale"])
    d = 2.0 ** -16 * scale * float((w.k[keys, kh].abs() @ q[i, h].abs()).max())
    tol = 2.0 ** -8 * want.abs() + (np.expm1(2 * d) + 2.0 ** -10 + 2.0 ** -14) * size + w.k[keys].shape[0] * 2.0 ** -33 * w.v[keys, kh].abs().max()
    off = (got[i, h] - want).abs() - tol
    assert bool((off <= 0).all()), (i, h, float(off.max()), got[i, h, :4], want[:4])


@pytest.mark.parametrize("new,copies,L", [(*FEW, 700), (*FEW, 9000), (3, 40, 300), (*MANY, 700), (300, 1, 9000)])      # whole keys and cut ones, in both kernels
@pytest.mark.parametrize("dim,size", [(128, 2.0 ** 126), (64, 1e33), (256, 1e35), (128, 1e-33), (64, 2.0 ** -116), (128, 2.0 ** -120)])
def test_sums_of_values_keep_the_values_range(torch, KV, dim, size, new, copies, L):
    """Values about as large, or as small, as 16-bit numbers are: their mean is a number like them, though their sum need not be."""
    w = Sequence(torch, KV, normal(torch, 9, L, 1, dim), (normal(torch, 10, L, 1, dim).clamp(-4, 4) * 0.1 + 1) * size)
    got, q = w.attend(normal(torch, 11, new, 4, dim), copies)
    for i in {0, 1, new - 1} & set(range(new)):
        close(w, got, q, i, i % 4)


def close_by_block(w, got, q, i, h, **kw):
    """As close(), where scales are so far apart that every block of 32 keys counts by itself: what may be left out is below 2^-33 of the largest weight in its block."""
    torch = w.torch
    keys, kh = w.seen(i, q.shape[0], kw.get("causal", True), kw.get("window", 0)), h // (q.shape[1] // w.heads)
    scale = w.D ** -0.5 if kw.get("scale") is None else abs(kw["scale"])
    k, v = w.k[keys, kh], w.v[keys, kh]
    p = torch.softmax(k @ q[i, h] * scale, 0)
    d = 2.0 ** -16 * scale * float((k.abs() @ q[i, h].abs()).max())
    # of a weight: twice the error of its exponent, rounding to 11 bits, fp32 sums and factors; of the sum of weights the same, on what the row is
    want = p @ v
    tol = 2.0 ** -8 * want.abs() + (np.expm1(2 * d) + 2.0 ** -10 + 2.0 ** -14) * (p @ v.abs())
    block = torch.arange(keys.start, keys.stop) // 32
    for b in block.unique():
        at = block == b
        tol = tol + 32 * 2.0 ** -33 * p[at].max() * v[at].abs().max()
    off = (got[i, h] - want).abs() - tol
    assert bool((off <= 0).all()), (i, h, float(off.max()), got[i, h, :4], want[:4])


LENGTHS = [(*FEW, 700), (*FEW, 9000), (8, 1, 2500), (3, 40, 300), (*MANY, 300), (*MANY, 6000), (300, 1, 9000)]


@pytest.mark.parametrize("new,copies,L", LENGTHS)
@pytest.mark.parametrize("dim,e", [(64, 18), (128, 30), (128, 40), (128, 100), (256, 60)])
def test_loud_values_that_a_row_does_not_see_do_not_matter_to_it(torch, KV, dim, e, new, copies, L):
    """Values are 2^e louder from the last block of 32 on that is the second of its 64; tokens before them do not see them.  The last tokens do."""
    v, start = normal(torch, 12, L, 1, dim), (L - 33) // 64 * 64 + 32
    v[start:] *= 2.0 ** e
    w = Sequence(torch, KV, normal(torch, 13, L, 1, dim), v * 2.0 ** -20)
    got, q = w.attend(normal(torch, 14, new, 4, dim), copies)
    first = start - (L - new)      # that sees them
    for i in {0, 1, new // 2, first - 40, first - 33, first - 20, first - 1, first, new - 1} & set(range(new)):
        close_by_block(w, got, q, i, i % 4)


@pytest.mark.parametrize("new,copies,L", LENGTHS)
@pytest.mark.parametrize("dim,e,window", [(64, 30, 40), (128, 40, 70), (128, 90, 120), (256, 40, 64)])
def test_loud_values_outside_a_row_s_window_do_not_matter_to_it(torch, KV, dim, e, window, new, copies, L):
    """Every third block is louder, so that windows begin and end in them."""
    v = normal(torch, 15, L, 1, dim)
    v[torch.arange(L) // 32 % 3 == 1] *= 2.0 ** e
    w = Sequence(torch, KV, normal(torch, 16, L, 1, dim), v * 2.0 ** -20)
    got, q = w.attend(normal(torch, 17, new, 4, dim), copies, window=window)
    for i in set(list(range(0, new, 13)) + [1, new - 2, new - 1]) & set(range(new)):
        close_by_block(w, got, q, i, i % 4, window=window)


@pytest.mark.parametrize("new,copies,L", LENGTHS)
@pytest.mark.parametrize("dim,e,below", [(64, 40, 300.0), (128, 40, 27.7), (128, 24, 16.6), (128, 100, 69.3), (256, 60, 41.6)])
@pytest.mark.parametrize("first", [True, False])
def test_loud_values_count_by_their_weight(torch, KV, first, dim, e, below, new, copies, L):
    """Values 2^e louder with scores `below` under the others: of no weight, or of so little that both sides count, before the others or behind them."""
    k, v, q = normal(torch, 18, L, 1, dim) * 0.25, normal(torch, 19, L, 1, dim), normal(torch, 20, new, 2, dim) * 0.25
    k[:, 0, 0] = 0.0
    q[..., 0] = 8.0
    at = (L - new) // 64 * 64 - 64      # (blocks of 32: what is quiet in one with loud values is held as next to nothing)
    at = slice(0, 64) if first else slice(at, at + 32)
    k[at, 0, 0] = -below * dim ** 0.5 / 8.0
    v[at] *= 2.0 ** e
    w = Sequence(torch, KV, k, v * 2.0 ** -20)
    got, q = w.attend(q, copies)
    for i in {0, new // 2, new - 1}:
        close_by_block(w, got, q, i, i % 2)


@pytest.mark.parametrize("new,copies,L", LENGTHS)
@pytest.mark.parametrize("up", [True, False])
def test_values_that_grow_or_fade_over_the_whole_range(torch, KV, up, new, copies, L):
    run = 2.0 ** torch.linspace(-118, 118, L)[:, None, None]
    w = Sequence(torch, KV, normal(torch, 21, L, 1, 128), normal(torch, 22, L, 1, 128) * (run if up else run.flip(0)))
    got, q = w.attend(normal(torch, 23, new, 2, 128), copies)
    for i in set(range(0, new, 17)) | {new - 1}:
        close_by_block(w, got, q, i, i % 2)


@pytest.mark.parametrize("new,copies,L", [(*FEW, 700), (*FEW, 9000), (*MANY, 300), (*MANY, 6000), (300, 1, 9000)])
def test_far_scales_with_vectors_that_are_not_finite_and_blocks_of_zeros(torch, KV, new, copies, L):
    """NaN for the rows that see the token, no others; zeros beside loud values stay zeros."""
    k, v = normal(torch, 24, L, 1, 64), normal(torch, 25, L, 1, 64)
    v[torch.arange(L) // 32 % 2 == 0] *= 2.0 ** 50
    v[32 * 3:32 * 5] = 0.0
    at = L - new // 2 - 1
    v[at, 0, 7] = float("nan")
    w = Sequence(torch, KV, k, v)
    got, q = w.attend(normal(torch, 26, new, 2, 64), copies)
    seeing = torch.arange(new) + L - new >= at
    assert torch.equal(torch.isnan(got).all(-1).all(-1), seeing) and not bool(torch.isnan(got[~seeing]).any())
    for i in {0, new // 4} & set(torch.nonzero(~seeing).flatten().tolist()):
        close_by_block(w, got, q, i, 0)


@pytest.mark.parametrize("dim,group", [(64, 4), (128, 2)])
def test_the_weights_that_are_summed_are_those_that_are_multiplied(torch, KV, dim, group):
    """Values of one have a mean of one, however the weights are rounded: of every chunk of the keys to what fp32 sums are off by.  (What the rounding of weights alone
    leaves is 2^-12 where one key outweighs the others, too little to be seen in 16 bits.)"""
    L = 9000
    w = Sequence(torch, KV, normal(torch, 27, L, 1, dim) * 3, torch.ones(L, 1, dim))
    batch = KV.KVBatch(w.i32([0, 1]), w.i32([L]), w.table, 1, 1, L)
    workspace = w.cache.attention_workspace(batch, group).zero_()
    w.attend(normal(torch, 28, 1, group, dim), workspace=workspace)
    part = group * (dim + 2)      # floats of a chunk: means of the rows, then their maxima and sums
    parts = workspace.view(torch.float32)[:20 * part].view(20, part)[:, :group * dim].double()
    assert float((parts - 1).abs().max()) <= 2.0 ** -18


@pytest.mark.parametrize("new,copies,L", [(*FEW, 300), (*FEW, 9000), (*MANY, 300), (300, 1, 9000)])
@pytest.mark.parametrize("apart", [False, True])
def test_large_channels_of_queries_where_keys_have_none(torch, KV, apart, new, copies, L):
    """Queries of 1e30 and keys of 1e17 in different channels: every score is zero, though the product of their scales is past fp32.  (apart: blocks of 32 by themselves.)"""
    k, q, v = torch.zeros(L, 1, 64), torch.zeros(new, 4, 64), normal(torch, 29, L, 1, 64)
    k[:, :, 7], q[:, :, 9] = 1e17, 1e30
    v[torch.arange(L) // 32 % 2 == 1] *= 2.0 ** (30 if apart else 1)
    w = Sequence(torch, KV, k, v)
    got, q = w.attend(q, copies)
    for i in {0, new // 2, new - 1}:
        (close_by_block if apart else close)(w, got, q, i, i % 4)
