"""Pages that sequences share: counts, tables and copies entry by entry against the oracle's, and what the sequences hold through forks, steps of their own, cuts and ends."""
import numpy as np
import pytest

from oracle import kv_stream_oracle as W
from paper_2411_05007_amd import svdq as S
from tests.test_gpu_kv_streams import DEV, Stream, i32

pytestmark = pytest.mark.gpu


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


class Pool:
    """A pool with tables on the GPU, the oracle's beside it, and caches whose bytes say what every token of every sequence is."""

    def __init__(self, torch, KV, pages, P, heads=2, dim=64, layers=1, seed=0):
        self.torch, self.KV, self.P, self.rng = torch, KV, P, np.random.default_rng(seed)
        self.pool, self.model = KV.KVPages(pages, P), W.Pages(pages, P)
        self.caches = [KV.KVCache(pages, heads, dim, P) for _ in range(layers)]
        for c in self.caches:
            for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales):
                t.copy_(torch.from_numpy(self.rng.integers(0, 255, t.shape, dtype=np.uint8)))
        self.shadow = [[t.cpu().numpy().copy() for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales)] for c in self.caches]

    def check(self, *tables):
        self.torch.cuda.synchronize()
        assert self.pool.refs.tolist() == self.model.refs
        for dev, host in tables:
            assert dev.tolist() == host
        for c, s in zip(self.caches, self.shadow):
            assert all(np.array_equal(t.cpu().numpy(), x) for t, x in zip((c.k_codes, c.k_scales, c.v_codes, c.v_scales), s))

    def reserve(self, dev, host, new, lens, **kw):
        cu = np.concatenate([[0], np.cumsum(new)])
        batch = self.KV.KVBatch(i32(self.torch, cu), i32(self.torch, lens), dev, int(cu[-1]), int(max(new, default=0)), int(max(lens, default=0)))
        missing = i32(self.torch, [77])
        self.pool.reserve(self.caches if len(self.caches) != 1 else self.caches[0], batch, missing, **kw)
        copies, lacks = self.model.reserve(host, new, lens)
        for s in self.shadow:
            for g, to, tokens in copies:
                if g >= 0:
                    for x in s:
                        x[to, :, :(tokens + 31) // 32] = x[g, :, :(tokens + 31) // 32]
        assert missing.tolist() == [lacks]
        return lacks


def empty(torch, B, width):
    return torch.full((B, width), -1, dtype=torch.int32, device=DEV), [[-1] * width for _ in range(B)]


@pytest.mark.parametrize("P,pages,B,width,layers", [(64, 25, 4, 9, 1), (32, 120, 7, 70, 2), (1024, 6, 3, 3, 1), (128, 3000, 33, 130, 1), (64, 70000, 150, 20, 0), (32, 5000, 700, 5, 0)])
def test_a_life_of_sequences_that_share_pages(torch, KV, P, pages, B, width, layers):
    """Prompts, forks, steps, cuts, ends, in any order, with shortages."""
    w = Pool(torch, KV, pages, P, layers=layers, seed=P + pages)
    rng, most = w.rng, width * P
    dev, host = zip(*(empty(torch, B, width) for _ in range(2)))
    lens = [[0] * B, [0] * B]
    short = 0
    for step in range(40):
        side = int(rng.integers(2))
        d, h = dev[side], host[side]
        what = rng.choice(["grow", "grow", "step", "step", "fork", "cut", "end", "window"])
        if what in ("grow", "step"):
            new = [int(min(most - n, 1 if what == "step" else rng.integers(0, min(most, 20 * P)))) for n in lens[side]]
            lens[side] = [n + m for n, m in zip(lens[side], new)]
            short += w.reserve(d, h, new, lens[side]) > 0
        elif what == "fork":
            other = 1 - side
            w.pool.release(dev[other])
            w.model.release(host[other])
            parent = rng.integers(-1, B + 1, B).tolist()
            out = i32(torch, [9] * B)
            w.pool.fork(d, i32(torch, lens[side]), i32(torch, parent), dev[other], out)
            w.model.fork(h, lens[side], parent, host[other], lens[other])
            assert out.tolist() == lens[other]
        elif what == "cut":
            lens[side] = [int(rng.integers(0, n + 1)) for n in lens[side]]
            w.pool.release(d, i32(torch, lens[side]))
            w.model.release(h, lens[side])
        elif what == "end":
            first = [0 if rng.random() < 0.3 else 2 ** 31 - 1 for _ in range(B)]
            lens[side] = [n if f else 0 for n, f in zip(lens[side], first)]
            w.pool.release(d, i32(torch, first))
            w.model.release(h, first)
        else:      # what a window left
            first, end = [int(rng.integers(0, 100)) for _ in range(B)], [max(0, n - 2 * P) for n in lens[side]]
            w.pool.release(d, i32(torch, first), i32(torch, end))
            w.model.release(h, first, end)
        w.check(*zip(dev, host))
    assert sum(w.model.refs) == sum(g >= 0 for h in host for row in h for g in row)
    assert short or pages > 2000


def test_more_entries_than_a_round_and_pages_far_apart(torch, KV):
    w = Pool(torch, KV, 66000, 32, layers=0)
    busy = np.ones(66000, np.int32)
    busy[w.rng.permutation(66000)[:1500]] = 0
    busy[65990:] = 0
    w.pool.refs.copy_(torch.from_numpy(busy))
    w.model.refs = busy.tolist()
    dev, host = empty(torch, 3, 900)
    lens = [0, 0, 0]
    for new in ([20, 32 * 700, 0], [32 * 3, 1, 32 * 600], [1, 31, 40], [32 * 300, 0, 32 * 100]):
        lens = [a + b for a, b in zip(lens, new)]
        w.reserve(dev, host, new, lens)
        w.check((dev, host))


def test_pages_are_private_before_they_are_written(torch, KV):
    """Three branches of a sequence in the middle of a block append their own tokens: each attends to its own, the parent keeps its."""
    H, D, P = 2, 128, 64
    w = Stream(torch, KV, H, D, P, [400], 3, q_heads=4, dims=D)
    pool = KV.KVPages(w.pages, P)
    table, length = i32(torch, np.full((1, 7), -1)), i32(torch, [0])
    gen = torch.Generator(device=DEV).manual_seed(5)
    rows = lambda n: torch.randn(n, 4 + 2 * H, D, generator=gen, device=DEV).to(torch.bfloat16)
    sent = {}

    def step(table, lens, x, new):
        cu = np.concatenate([[0], np.cumsum(new)])
        batch = KV.KVBatch(i32(torch, cu), i32(torch, lens), table, int(cu[-1]), max(new), max(lens))
        missing = i32(torch, [5])
        pool.reserve(w.cache, batch, missing)
        assert missing.item() == 0
        w.cache.append(x[:, 4:4 + H], x[:, 4 + H:], batch, w.rope)
        return w.cache.attention(x[:, :4], batch, w.rope)
    prompt = rows(150)
    step(table, [150], prompt, [150])
    branch, lens = i32(torch, np.full((3, 7), -1)), i32(torch, [0] * 3)
    pool.fork(table, i32(torch, [150]), i32(torch, [0, 0, 0]), branch, lens)
    assert lens.tolist() == [150] * 3 and sorted(pool.refs.tolist())[-3:] == [4, 4, 4]
    own = [rows(90) for _ in range(3)]
    at = [0, 0, 0]
    for n in (1, 5, 84):
        out = step(branch, [150 + a + n for a in at], torch.cat([own[b][at[b]:at[b] + n] for b in range(3)]), [n] * 3)
        at = [a + n for a in at]
    assert len(set(branch[:, 2].tolist())) == 3 and branch[:, :2].unique(dim=0).shape[0] == 1
    # alone, the same tokens in the same calls
    for b in range(3):
        w2 = Stream(torch, KV, H, D, P, [400], 4, q_heads=4, dims=D)
        t2, done = i32(torch, w2.table), 0
        for part in (prompt, own[b][:1], own[b][1:6], own[b][6:]):
            done += len(part)
            batch = KV.KVBatch(i32(torch, [0, len(part)]), i32(torch, [done]), t2, len(part), len(part), done)
            w2.cache.append(part[:, 4:4 + H], part[:, 4 + H:], batch, w2.rope)
        want = w2.cache.attention(own[b][6:, :4], batch, w2.rope)
        assert float((out[84 * b:84 * b + 84].float() - want.float()).abs().max()) <= 2.0 ** -7 * float(want.float().abs().max())      # (another cut of the rows)
        for x, y in zip(w.cache.gather(KV.KVRows(i32(torch, [0]), i32(torch, [0, 240]), branch[b:b + 1].contiguous(), 240)),
                        w2.cache.gather(KV.KVRows(i32(torch, [0]), i32(torch, [0, 240]), t2, 240))):
            assert torch.equal(x, y)
    pool.release(branch)
    pool.release(table)
    assert not pool.refs.any() and (table == -1).all() and (branch == -1).all()


def test_entries_out_of_range_name_no_page(torch, KV):
    w = Pool(torch, KV, 10, 32)
    dev, host = empty(torch, 4, 3)
    odd = [[-7, 10, 2 ** 31 - 1], [-2 ** 31, 3, -1], [4, 4, 11], [0, 1, 2]]
    dev.copy_(i32(torch, odd))
    host = [list(r) for r in odd]
    w.pool.refs.copy_(i32(torch, [1, 1, 1, 1, 2, 0, 0, 0, 0, 0]))
    w.model.refs = w.pool.refs.tolist()
    lens = [2 ** 31 - 1, -5, 96, 40]
    out, hl = i32(torch, [0] * 4), [0] * 4
    to, ho = empty(torch, 4, 2)      # (narrower)
    w.pool.fork(dev, i32(torch, lens), i32(torch, [0, 1, 3, 2]), to, out)
    w.model.fork(host, lens, [0, 1, 3, 2], ho, hl)
    assert out.tolist() == hl == [64, 0, 40, 64]
    w.check((dev, host), (to, ho))
    w.reserve(to, ho, [5, 3, 2, 33], [64, 0, 2 ** 31 - 1, 31])
    w.check((dev, host), (to, ho))
    w.pool.release(dev, i32(torch, [-2 ** 31, 0, 1, 2 ** 31 - 1]), i32(torch, [2 ** 31 - 1, 31, 64, 5]))
    w.model.release(host, [-2 ** 31, 0, 1, 2 ** 31 - 1], [2 ** 31 - 1, 31, 64, 5])
    w.check((dev, host), (to, ho))
    w.pool.release(dev)
    w.model.release(host)
    w.check((dev, host), (to, ho))
    # counts of tokens that do not ascend, no tokens, no sequences
    for cu in ([0, 60, 20, 20, 90], [-5, 400, 7, 8, 9]):
        batch = KV.KVBatch(i32(torch, cu), i32(torch, [30, 20, 10, 64]), to, 90, 90, 64)
        w.pool.reserve(w.caches[0], batch)
    missing = i32(torch, [3])
    w.pool.reserve(w.caches[0], KV.KVBatch(i32(torch, [0]), i32(torch, []), to[:0], 0, 0, 0), missing)
    assert missing.item() == 0
    missing.fill_(3)
    before = to.clone(), w.pool.refs.clone()
    w.pool.reserve(w.caches[0], KV.KVBatch(i32(torch, [0] * 5), i32(torch, [30] * 4), to, 0, 0, 30), missing)
    assert missing.item() == 0 and torch.equal(before[0], to) and torch.equal(before[1], w.pool.refs)


@pytest.mark.parametrize("dim,heads,P", [(64, 1, 32), (128, 3, 64), (256, 2, 1024)])
def test_pages_are_copied_between_caches(torch, KV, dim, heads, P):
    a, b = Pool(torch, KV, 6, P, heads, dim, seed=1), Pool(torch, KV, 9, P, heads, dim, seed=2)
    copies = [(0, 8, P), (5, 0, 1), (3, 1, 33 if P > 32 else 0), (2, 2, 2 ** 31 - 1), (-1, 3, 5), (6, 4, 5), (1, 9, 5), (1, -1, 5), (4, 5, -3), (4, 6, 0), (2 ** 31 - 1, 7, P)]
    b.caches[0].copy_pages(i32(torch, copies), source=a.caches[0])
    for g, to, n in copies:
        if 0 <= g < 6 and 0 <= to < 9 and n > 0:
            for x, y in zip(b.shadow[0], a.shadow[0]):
                x[to, :, :(n + 31) // 32] = y[g, :, :(n + 31) // 32]
    a.check()
    b.check()
    a.caches[0].copy_pages(i32(torch, np.zeros((0, 3))))
    a.caches[0].copy_pages(i32(torch, [(0, 1, P), (2, 3, P)]))      # within one cache
    for x in a.shadow[0]:
        x[1], x[3] = x[0], x[2]
    a.check()


@pytest.mark.parametrize("pages,P", [(9, 64), (10, 32), (10, 128)])
def test_caches_that_do_not_fit_the_pool_are_refused_before_anything_is_changed(torch, KV, pages, P):
    w = Pool(torch, KV, 10, 64)
    dev, host = empty(torch, 1, 4)
    other = KV.KVCache(pages, 2, 64, P)
    for caches in ([w.caches[0], other], [other, w.caches[0]], other):      # (a further layer's as well as the first one's)
        with pytest.raises(AssertionError):
            w.pool.reserve(caches, KV.KVBatch(i32(torch, [0, 70]), i32(torch, [70]), dev, 70, 70, 70))
    w.check((dev, host))


def test_branches_in_a_captured_step(torch, KV):
    """Release, fork, reserve and append in one graph, replayed with other parents and with eager work between: every replay as the eager calls."""
    B, P, H, D = 6, 64, 2, 64
    worlds = []
    for _ in range(2):
        w = Pool(torch, KV, 80, P, H, D, layers=2, seed=8)
        dev, host = empty(torch, 2, 8)
        lens = [300, 129]
        w.reserve(dev, host, lens, lens)
        to, ho = empty(torch, B, 8)
        state = dict(w=w, table=dev, length=i32(torch, lens), to=to, out=i32(torch, [0] * B), parent=i32(torch, [0] * B), missing=i32(torch, [0]),
                     x=torch.randn(B, 2 * H, D, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(torch.bfloat16), one=i32(torch, [1] * B))
        state["batch"] = KV.KVBatch(i32(torch, range(B + 1)), state["out"], to, B, 1, 512)
        state["ws"] = w.pool.reserve_workspace(state["batch"])
        worlds.append(state)

    def step(s):
        w = s["w"]
        w.pool.release(s["to"])
        w.pool.fork(s["table"], s["length"], s["parent"], s["to"], s["out"])
        s["out"].add_(s["one"])
        w.pool.reserve(w.caches, s["batch"], s["missing"], workspace=s["ws"])
        for c in w.caches:
            c.append(s["x"][:, :H], s["x"][:, H:], s["batch"])
    eager, graphed = worlds
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(graphed)
    torch.cuda.current_stream().wait_stream(side)
    step(eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed)
    rng = np.random.default_rng(2)
    for i in range(8):
        parent = i32(torch, rng.integers(-1, 3, B))
        for s in worlds:
            s["parent"].copy_(parent)
            s["x"].mul_(1.5)
        graph.replay()
        step(eager)
        torch.cuda.synchronize()
        for k in ("to", "out", "missing"):
            assert torch.equal(eager[k], graphed[k]), (i, k)
        assert torch.equal(eager["w"].pool.refs, graphed["w"].pool.refs) and eager["missing"].item() == 0
        for a, b in zip(eager["w"].caches, graphed["w"].caches):
            for n in ("k_codes", "k_scales", "v_codes", "v_scales"):
                assert torch.equal(getattr(a, n), getattr(b, n)), (i, n)


def test_the_pool_on_another_stream(torch, KV):
    w = Pool(torch, KV, 40, 64)
    dev, host = empty(torch, 3, 6)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    w.reserve(dev, host, [100, 5, 0], [100, 5, 0], stream=stream)
    to, ho = empty(torch, 4, 6)
    out, hl = i32(torch, [0] * 4), [0] * 4
    args = i32(torch, [100, 5, 0]), i32(torch, [0, 0, 1, 2])
    stream.wait_stream(torch.cuda.current_stream())
    w.pool.fork(dev, *args, to, out, stream=stream)
    w.model.fork(host, [100, 5, 0], [0, 0, 1, 2], ho, hl)
    stream.synchronize()
    w.reserve(to, ho, [30, 1, 2, 3], [130, 101, 7, 3], stream=stream)
    stream.synchronize()
    w.check((dev, host), (to, ho))
    w.pool.release(to, stream=stream)
    w.model.release(ho)
    stream.synchronize()
    w.check((dev, host), (to, ho))
