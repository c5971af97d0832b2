"""Pages after a shortage: what a sequence could not write it never sees, whoever's pages it gets later, and what it does see is its own.  The tokens that a row of a table holds are
kept on the host, token by token; attention is held to the definition in 64 bits over those alone."""
import numpy as np
import pytest

from oracle import kv_oracle as K
from oracle import kv_stream_oracle as W
from paper_2411_05007_amd import svdq as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


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


def i32(torch, x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


class World:
    """Rows of tables on a pool whose free pages hold loud tokens of nobody.  Beside a table: host, its rows as the oracle has them; lens; have, the tokens that a row holds; sent, what
    was appended for each."""

    def __init__(self, torch, KV, pages, P=64, H=2, G=2, D=64, seed=0):
        self.torch, self.KV, self.P, self.H, self.G, self.D = torch, KV, P, H, G, D
        self.rng = np.random.default_rng(seed)
        self.cache, self.pool, self.model = KV.KVCache(pages, H, D, P), KV.KVPages(pages, P), W.Pages(pages, P)
        for codes, scales in ((self.cache.k_codes, self.cache.k_scales), (self.cache.v_codes, self.cache.v_scales)):
            codes.copy_(torch.from_numpy(self.rng.integers(0, 0x78, codes.shape, dtype=np.uint8)))
            scales.fill_(127)      # (up to 240)
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        self.missing = i32(torch, [0])

    def rows(self, n, width):
        t = self.torch.full((n, width), -1, dtype=self.torch.int32, device=DEV)
        t.host, t.have, t.sent, t.lens = [[-1] * width for _ in range(n)], [set() for _ in range(n)], [{} for _ in range(n)], [0] * n
        return t

    def batch(self, table, new, lens=None):
        cu = np.concatenate([[0], np.cumsum(new)])
        n = table.lens if lens is None else lens
        return self.KV.KVBatch(i32(self.torch, cu), i32(self.torch, n), table, int(cu[-1]), max(int(max(new)), 1), table.shape[1] * self.P)

    def fork(self, table, parent, to):
        out = i32(self.torch, [0] * to.shape[0])
        self.pool.fork(table, i32(self.torch, table.lens), i32(self.torch, parent), to, out)
        self.model.fork(table.host, table.lens, parent, to.host, to.lens)
        assert out.tolist() == to.lens and to.tolist() == to.host
        to.have, to.sent = [set(table.have[p]) for p in parent], [dict(table.sent[p]) for p in parent]

    def release(self, table, first):
        """first: of each row, the first token that goes; None: of that row none"""
        first = [2 ** 31 - 1 if f is None else f for f in first]
        self.pool.release(table, i32(self.torch, first))
        self.model.release(table.host, first)
        for b, row in enumerate(table.host):
            table.have[b] = {t for t in table.have[b] if row[t // self.P] >= 0}

    def end(self, *ends):
        """(table, row): gives back what it has"""
        for table, b in ends:
            self.release(table, [0 if i == b else None for i in range(table.shape[0])])
            table.lens[b] = 0

    def random(self, n, scale=1.0):
        return (self.torch.randn(n, (self.G + 2) * self.H, self.D, generator=self.gen, device=DEV) * scale).to(self.torch.bfloat16)

    def launch(self, x, batch, out=None, pages=None, workspace=None):
        Q = self.G * self.H
        self.pool.reserve(self.cache, batch, self.missing, workspace=pages)
        self.cache.append(x[:, Q:Q + self.H], x[:, Q + self.H:], batch)
        return self.cache.attention(x[:, :Q], batch, out=out, workspace=workspace)

    def step(self, table, new, scale=1.0):
        table.lens = [a + b for a, b in zip(table.lens, new)]
        x = self.random(sum(new), scale)
        out = self.launch(x, self.batch(table, new))
        return self.look(table, new, x, out)

    def look(self, table, new, x, out):
        """Counts the new tokens in where they have a page, holds `out` to what the rows see, then tables and counts to the oracle's; returns how many entries got no page."""
        self.torch.cuda.synchronize()
        pages, xn, got, Q, at0 = table.tolist(), x.float().cpu().numpy().astype(np.float64), out.float().cpu().numpy().astype(np.float64), self.G * self.H, 0
        for b, n in enumerate(new):
            at = table.lens[b] - n + np.arange(n)
            table.have[b] = {t for t in table.have[b] if pages[b][t // self.P] >= 0} | {int(t) for t in at if pages[b][t // self.P] >= 0}
            table.sent[b].update({int(t): xn[at0 + i, Q:] for i, t in enumerate(at)})
            if n:
                keys = np.array(sorted(table.have[b]), np.int64)
                k, v, kb, vb = self.held(pages[b], keys)
                for y, held, byte in ((0, k, kb), (self.H, v, vb)):      # what was appended, within its own block's scale
                    want = np.array([table.sent[b][t][y:y + self.H] for t in keys]).reshape(held.shape)
                    s = np.exp2(np.maximum(byte, 1) - 127.0)[..., None]
                    assert (np.abs(held - want) <= W.code_bounds(want, 0.0, byte[..., None]) + 2.0 ** -10 * s).all(), b      # (rounded again where the scale grew)
                q = xn[at0:at0 + n, :Q]
                want, tol = W.attention(q, np.abs(q), k, v, at, keys, self.D ** -0.5)
                assert (np.abs(got[at0:at0 + n] - want) <= tol).all(), (b, at[0], float(np.abs(got[at0:at0 + n] - want).max()))
            at0 += n
        _, missing = self.model.reserve(table.host, new, table.lens)
        assert table.tolist() == table.host and self.pool.refs.tolist() == self.model.refs and self.missing.item() == missing
        return missing

    def held(self, row, keys):
        kc, ks, vc, vs = (t.cpu().numpy() for t in (self.cache.k_codes, self.cache.k_scales, self.cache.v_codes, self.cache.v_scales))
        shape = (len(keys), self.H)
        k, v, kb, vb = np.zeros(shape + (self.D,)), np.zeros(shape + (self.D,)), np.zeros(shape, np.int64), np.zeros(shape, np.int64)
        blocks = {}
        for i, t in enumerate(keys):
            page, at = row[t // self.P], t % self.P // 32
            for h in range(self.H):
                kb[i, h], vb[i, h] = ks[page, h, at], vs[page, h, at]
                if (page, h, at) not in blocks:
                    blocks[page, h, at] = K.block_numbers(kc[page, h, at], vc[page, h, at])
                a, b = blocks[page, h, at]
                k[i, h], v[i, h] = a[t % 32] * 2.0 ** (kb[i, h] - 127), b[t % 32] * 2.0 ** (vb[i, h] - 127)
        return k, v, kb, vb

    def bytes_are_their_own(self, table, b):
        """Every block's scale byte is that of what the row appended there (a row that took over nothing)."""
        keys = np.array(sorted(table.have[b]))
        _, _, kb, vb = self.held(table.tolist()[b], keys)
        for blk in set((keys // 32).tolist()):
            here = keys // 32 == blk
            sent = np.array([table.sent[b][t] for t in keys[here]])
            for h in range(self.H):
                assert (kb[here, h] == K.scale_byte(np.abs(sent[:, h]).max())).all() and (vb[here, h] == K.scale_byte(np.abs(sent[:, self.H + h]).max())).all(), (b, blk, h)


@pytest.mark.parametrize("P,D,new", [(64, 64, [5, 1, 0, 7, 1, 40, 8, 5, 1, 30, 1]), (32, 128, [1, 1, 0, 1, 20, 7, 40, 1, 1, 2]), (128, 64, [128, 1, 0, 126, 1, 1, 3]), (64, 256, [100, 3, 0, 20, 1, 9, 60, 1])])
def test_a_page_shows_nothing_of_its_last_owner(torch, KV, P, D, new):
    """Sequence 1 finds the pool dry, sequence 0 ends (where the list has 0), 1 goes on in pages that 0 had: the tokens that were not written stay unseen."""
    w = World(torch, KV, 3, P, D=D, seed=P + D)
    t = w.rows(2, 6)
    assert w.step(t, [3 * P, 0], scale=8.0) == 0
    for n in new:
        if n == 0:
            w.end((t, 0))
        else:
            w.step(t, [0, n], scale=0.01)
    w.bytes_are_their_own(t, 1)
    dry = sum(new[:new.index(0)])      # tokens that found the pool dry, and those behind them in the last one's page
    assert t.have[1] == set(range((dry + P - 1) // P * P, sum(new)))
    w.end((t, 1))
    assert not w.pool.refs.any()


def test_a_captured_step_goes_on_after_a_shortage(torch, KV):
    """One token of each a replay; no host looks at what is missing, but the count of a step can be added up on the GPU."""
    P = 32
    w = World(torch, KV, 4, P, seed=3)
    t = w.rows(2, 5)
    w.step(t, [64, 64], scale=8.0)      # the pool is dry
    length, one, total = i32(torch, t.lens), i32(torch, [1, 1]), i32(torch, [0])
    batch = KV.KVBatch(i32(torch, [0, 1, 2]), length, t, 2, 1, 5 * P)
    x, out = w.random(2), torch.empty(2, w.G * w.H, w.D, dtype=torch.bfloat16, device=DEV)
    pages, ws = w.pool.reserve_workspace(batch), w.cache.attention_workspace(batch, w.G * w.H)
    idle = KV.KVBatch(i32(torch, [0] * 3), i32(torch, [0] * 2), torch.full_like(t, -1), 2, 1, 5 * P)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):      # (the first call of a kernel loads it)
        w.launch(x, idle, out, pages, ws)
        total.add_(w.missing)
        length.add_(one)
        length.sub_(one)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        length.add_(one)
        w.launch(x, batch, out, pages, ws)
        total.add_(w.missing)
    lost = 0
    for i in range(70):
        if i == 5:      # sequence 0 ends and begins anew
            w.end((t, 0))
            length.copy_(i32(torch, [0, t.lens[1]]))
        x.copy_(w.random(2, 0.05))
        t.lens = [n + 1 for n in t.lens]
        graph.replay()
        lost += w.look(t, [1, 1], x, out)
        assert length.tolist() == t.lens and total.item() == lost
    # 0 and 1 without a third page; 1 to the end of its third; then 0 without its second and 1 without its fifth
    assert lost == 2 * 5 + 27 + 33 + 6 and 96 in t.have[1] and not t.have[1] & set(range(64, 96))


def test_a_branch_that_found_no_page_for_its_prefix(torch, KV):
    """Its parent keeps the page; what the branch's page would have held it never sees, what it adds behind that page it does."""
    P = 64
    w = World(torch, KV, 3, P, seed=4)
    t, c = w.rows(2, 4), w.rows(2, 4)
    w.step(t, [40, 0])
    w.step(t, [0, 128], scale=8.0)      # the pool is dry
    w.fork(t, [0, 0], c)
    assert w.step(c, [1, 0]) == 1 and c[0].tolist() == [-1] * 4 and c[1, 0] == t[0, 0]
    w.end((t, 1))
    for n in (1, 20):
        assert w.step(c, [n, 0]) == 1 and not c.have[0]
    assert w.step(c, [5, 0]) == 1 and sorted(c.have[0]) == [64, 65, 66]      # into its next page
    assert w.step(t, [3, 0]) == 0 and t[0, 0] != c[1, 0]      # (the other branch still names the page that the parent wrote in)
    w.end((c, 0), (c, 1), (t, 0))
    assert not w.pool.refs.any()


def test_a_page_that_was_given_back_under_its_tokens(torch, KV):
    """A row that gives back the page it stands in, and goes on: the tokens there are gone, and nothing stands in for them."""
    P = 64
    w = World(torch, KV, 4, P, seed=5)
    t = w.rows(2, 4)
    w.step(t, [70, 10])
    w.release(t, [64, None])
    assert w.step(t, [1, 1]) == 1 and t[0, 1] == -1 and len(t.have[0]) == 64
    assert w.step(t, [57, 1]) == 1 and t[0, 1] == -1 and len(t.have[0]) == 64
    assert w.step(t, [1, 1]) == 0 and sorted(t.have[0])[-1] == 128      # its next page


def test_a_reservation_that_is_tried_again(torch, KV):
    """A call that came up short and is repeated when there is room, lengths as they were, gets what it lacked where the page's first token is a new one."""
    P = 32
    w = World(torch, KV, 4, P, seed=6)
    t = w.rows(2, 6)
    w.step(t, [0, 64], scale=8.0)
    w.step(t, [20, 0])
    t.lens[0] = 20 + 70
    batch = w.batch(t, [70, 0])
    w.pool.reserve(w.cache, batch, w.missing)
    assert w.missing.item() == 1 and (t[0] >= 0).tolist() == [True, True, False, False, False, False]
    w.model.reserve(t.host, [70, 0], t.lens)
    w.end((t, 1))
    x = w.random(70)
    out = w.launch(x, batch)
    assert w.look(t, [70, 0], x, out) == 0 and t.have[0] == set(range(90))


# ---- the last holders of a page ------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("free", [0, 1])
def test_the_last_holders_of_a_page_leave_it_to_the_first_of_them(torch, KV, free):
    """Two branches of a prompt that has ended write beside each other: one keeps the page, the other copies it, or, in a full pool, is the only one that loses its tokens there."""
    P = 64
    w = World(torch, KV, 2 + free, P, seed=7)
    t, c = w.rows(2, 2), w.rows(2, 3)
    w.step(t, [40, 0])
    w.step(t, [0, 30], scale=8.0)
    w.fork(t, [0, 0], c)
    w.end((t, 0))
    for new in ([1, 1], [3, 0], [0, 5], [7, 9]):
        assert w.step(c, new) == (0 if free or new[1] == 0 else 1)
    assert c.have[0] == set(range(51)) and c.have[1] == (set(range(55)) if free else set())
    w.end((c, 0), (c, 1), (t, 1))
    assert not w.pool.refs.any()


def test_many_branches_that_outlive_their_prompt(torch, KV):
    """130 of them, cut back into a page that they share and past others; the first ones stand still for a while."""
    P, B = 32, 130
    w = World(torch, KV, 900, P, H=1, G=1, seed=8)
    t, c = w.rows(1, 8), w.rows(B, 8)
    w.step(t, [200])
    w.fork(t, [0] * B, c)
    w.end((t, 0))
    c.lens = [100 + b % 3 for b in range(B)]
    c.have = [{k for k in held if k < n} for held, n in zip(c.have, c.lens)]
    assert w.step(c, [0, 0] + [1 + b % 41 for b in range(2, B)]) == 0
    assert w.step(c, [1] * B) == 0 and c[0, 3] != c[1, 3]
    assert w.step(c, [5 * (b % 7) for b in range(B)]) == 0


@pytest.mark.parametrize("B", [3, 64, 65])
def test_the_page_of_a_prefix_in_a_captured_step(torch, KV, B):
    """Branches go on alone, a token of each a replay, and all take over another's tokens between two of them: as many pages as they need if one of them keeps what is shared."""
    P = 32
    w = World(torch, KV, B + 1, P, H=1, G=1, seed=9 + B)
    t, c = w.rows(1, 4), w.rows(B, 4)
    w.step(t, [45])
    w.fork(t, [0] * B, c)
    length = i32(torch, c.lens)
    batch = KV.KVBatch(i32(torch, range(B + 1)), length, c, B, 1, 4 * P)
    x, out, one = w.random(B), torch.empty(B, 1, w.D, dtype=torch.bfloat16, device=DEV), i32(torch, [1] * B)
    pages, ws = w.pool.reserve_workspace(batch), w.cache.attention_workspace(batch, 1)
    idle = KV.KVBatch(i32(torch, [0] * (B + 1)), i32(torch, [0] * B), torch.full_like(c, -1), B, 1, 4 * P)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):      # (the first call of a kernel loads it)
        w.launch(x, idle, out, pages, ws)
        length.add_(one)
        length.sub_(one)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        length.add_(one)
        w.launch(x, batch, out, pages, ws)
    w.end((t, 0))
    for i in range(4):
        if i == 2:      # everyone takes over the last one's tokens
            t2 = w.rows(B, 4)
            w.fork(c, [B - 1] * B, t2)
            w.end(*((c, b) for b in range(B)))
            w.fork(t2, list(range(B)), c)
            w.end(*((t2, b) for b in range(B)))
            length.copy_(i32(torch, c.lens))
        x.copy_(w.random(B))
        c.lens = [n + 1 for n in c.lens]
        graph.replay()
        assert w.look(c, [1] * B, x, out) == 0 and len(set(c[:, 1].tolist())) == B
