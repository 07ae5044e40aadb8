"""Attention over selected blocks on the device, against plain 64-bit forms
(MI355X only)."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2607_26475_amd as ckv
from blocks_helpers import attend64, block_there, landmarks64, poison, select64
from e2m1_helpers import Pool4
from paged_helpers import D, SCALE, Pool

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _log(*a):
    print(*a, flush=True)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def make(kind, lens, Hkv, page, **kw):
    return Pool4(lens, Hkv, page, **kw) if kind == "e2m1" else Pool(lens, Hkv, page, kind, **kw)


class Call:
    """The three operators over a pool with their outputs."""

    def __init__(self, pool, G, block, k, n):
        self.pool, self.block, self.k, self.shape = pool, block, k, pool.shape(G)
        nb = -(-pool.max_ctx // block)
        self.marks = torch.zeros((pool.B, pool.Hkv, nb, D), dtype=torch.bfloat16, device=DEV)
        self.idx = torch.full((n, pool.Hkv, k), 99, dtype=torch.int32, device=DEV)
        self.out = torch.full((n, G * pool.Hkv, D), 9.0, device=DEV)
        self.lse = torch.full((n, G * pool.Hkv), 9.0, device=DEV)
        self.ws = ckv.blocks_workspace(self.shape, block, k, n)
        self.ws.fill_(0xFF)

    def landmarks(self, first=None, stream=None):
        ckv.paged_landmarks(self.shape, self.pool.cache, self.block, self.pool.ctx, self.marks,
                            first=first, stream=stream)

    def select(self, req, pos, q, stream=None):
        ckv.select_blocks(self.shape, self.pool.cache, self.block, self.k, req, pos, q, self.marks,
                          self.idx, self.ws, stream=stream)

    def attend(self, req, pos, q, lse=True, stream=None):
        ckv.paged_block_attn(self.shape, self.pool.cache, self.block, self.k, req, pos, q, self.idx,
                             SCALE, self.out, self.lse if lse else None, self.ws, stream=stream)


def check(pool, G, block, k, tokens, seed=0):
    """All three against the plain forms (the selection's sets exactly)."""
    req, pos = [t[0] for t in tokens], [t[1] for t in tokens]
    q = torch.randn((len(tokens), G * pool.Hkv, D), generator=torch.Generator().manual_seed(seed))
    q = q.to(torch.bfloat16)
    c = Call(pool, G, block, k, len(tokens))
    r, p, qd = _i32(req), _i32(pos), q.to(DEV)
    c.landmarks()
    marks = landmarks64(pool, block)
    assert torch.equal(c.marks.cpu().double(), marks.double())
    c.select(r, p, qd)
    want = select64(pool, block, k, req, pos, q, marks)
    assert torch.equal(c.idx.cpu(), want)
    c.attend(r, p, qd)
    out, lse, tol = attend64(pool, block, req, pos, q, want)
    got, gl = c.out.cpu().double(), c.lse.cpu().double()
    none = lse == -math.inf
    assert torch.all(got[none] == 0) and torch.all(gl[none] == -math.inf)
    err = (got - out).abs().amax(-1)
    assert torch.all(err <= tol), float((err / tol.clamp(min=1e-30)).max())
    # the log-sum's error is its logits' and 2^-22 of its own size
    assert torch.all(((gl - lse).abs() <= tol + 2.0 ** -22 * lse.abs() + 1e-6)[~none])
    return c, r, p, qd


def ragged_tokens(lens, new):
    return [(b, p) for b, n in enumerate(lens) for p in range(max(0, n - new), n)]


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("page,order,block,G,k", [
    (16, "pairs", 32, 4, 4), (32, "heads", 64, 1, 8), (256, "rows", 64, 2, 3),
    (16, "heads", 128, 8, 2), (64, "rows", 256, 16, 2), (128, "pairs", 32, 16, 64)])
def test_a_ragged_prefill(kind, page, order, block, G, k):
    """Chunks of several requests, holes, an empty request, padding and bad tokens
    between them, a request's tokens apart from each other."""
    _log("blocks", kind, page, order, block, G, k)
    lens = [700, 1, 0, 33, 513]
    pool = make(kind, lens, 2, page, seed=G, order=order, holes=[(0, 1), (4, 0), (3, 0)],
                max_ctx=777)
    tokens = ragged_tokens(lens, 37)
    tokens = tokens[:11] + [(0, -1), (5, 3), (-1, 0), (1, 777)] + tokens[11:] + \
        [(4, 100), (0, 0), (4, 511), (0, 350)]
    check(pool, G, block, k, tokens, seed=page)


@pytest.mark.parametrize("kind", ["bf16", "e2m1"])
@pytest.mark.parametrize("n,k", [(1, 1), (31, 5), (32, 2), (33, 2), (1000, 1), (2500, 7)])
def test_one_token(kind, n, k):
    """Single tokens: lengths around a block, pieces of a list, no earlier block kept."""
    _log("one token", kind, n, k)
    pool = make(kind, [n], 1, 16, seed=n)
    for G in (1, 4, 16):
        check(pool, G, 32, k, [(0, n - 1)])


@pytest.mark.parametrize("B,G,k,block", [(7, 4, 16, 64), (40, 8, 40, 32), (3, 1, 64, 32)])
def test_a_decode_step(B, G, k, block):
    """One token of every request, without a request list."""
    lens = [3000 - 67 * b for b in range(B)]
    pool = make("e2m1", lens, 2, 64, seed=B, max_ctx=3001)
    c, r, p, q = check(pool, G, block, k, [(b, n - 1) for b, n in enumerate(lens)])
    out, idx = c.out.clone(), c.idx.clone()
    c.idx.fill_(99)
    c.select(None, p, q)
    c.attend(None, p, q, lse=False)
    assert torch.equal(c.idx, idx) and torch.equal(c.out, out)


def test_many_tokens_of_one_request():
    """Enough tokens for the scoring of four tiles a workgroup and one piece a tile."""
    pool = make("bf16", [2600], 4, 16, seed=3)
    check(pool, 1, 64, 6, ragged_tokens([2600], 1100))


@pytest.mark.parametrize("nb", [300, 1500, 3001, 4200])
def test_many_blocks(nb):
    """Scores held in 16, 32 and 64 registers a lane, and read again at each halving."""
    n = 32 * nb - 5
    pool = make("e2m1", [n, n - 1000], 1, 64, seed=nb)
    check(pool, 4, 32, 33, [(0, n - 1), (0, n // 2), (1, n - 1001), (1, 3), (0, 31), (0, 32)])


def test_equal_and_nearly_equal_landmarks():
    """Ties go to the lower block; sums that differ by less than fp32 sees are
    ranked by what they are."""
    block, nb, k = 32, 200, 9
    n = block * nb
    pool = make("bf16", [n], 1, 16, seed=1)
    g = torch.Generator().manual_seed(8)
    pos = [n - 1, n - 33, 700]
    q = torch.randn((3, 2, D), generator=g).to(torch.bfloat16)
    base = torch.randn(D, generator=g).to(torch.bfloat16)
    cases = [base.expand(nb, D).clone(), torch.zeros((nb, D), dtype=torch.bfloat16)]
    near = base.expand(nb, D).clone()  # the same but for one tiny element
    near[torch.arange(nb), torch.arange(nb) % D] = (
        2.0 ** -30 * torch.randn(nb, generator=g)).to(torch.bfloat16)
    cases.append(near)
    far = torch.randn((nb, D), generator=g).to(torch.bfloat16)
    far[::3] = far[0]                  # many equal among others
    cases += [far, 2.0 ** -70 * far, 2.0 ** 50 * far]
    big = far.clone()                  # large terms that cancel
    big[:, 0], big[:, 1] = 2.0 ** 20, 2.0 ** 20
    q[:, :, 1] = -q[:, :, 0]
    cases.append(big)
    c = Call(pool, 2, block, k, 3)
    for i, m in enumerate(cases):
        _log("case", i)
        marks = m[None, None].to(torch.bfloat16)
        c.marks.copy_(marks)
        c.select(_i32([0, 0, 0]), _i32(pos), q.to(DEV))
        assert torch.equal(c.idx.cpu(), select64(pool, block, k, [0, 0, 0], pos, q, marks)), i


def test_landmarks_that_are_no_numbers_are_not_selected():
    pool = make("bf16", [640], 1, 16, seed=2)
    c = Call(pool, 4, 32, 6, 1)
    marks = torch.randn((1, 1, 20, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    marks[0, 0, 3, 5] = float("nan")
    marks[0, 0, 19] = float("nan")     # its own: not read
    q = torch.randn((1, 4, D), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    c.marks.copy_(marks)
    c.select(_i32([0]), _i32([639]), q.to(DEV))
    assert torch.equal(c.idx.cpu(), select64(pool, 32, 6, [0], [639], q, marks))
    assert 3 not in c.idx[0, 0].tolist()


def test_landmarks_from_a_position_on():
    """Only the blocks from first on are written; none where nothing is there."""
    lens = [200, 64, 0, 130]
    pool = make("e4m3", lens, 2, 16, seed=5, holes=[(0, 12), (3, 0), (3, 1)], max_ctx=256)
    c = Call(pool, 1, 32, 1, 1)
    c.marks.fill_(3.0)
    first = [97, 64, 0, 500]
    c.landmarks(first=_i32(first))
    old = torch.full(c.marks.shape, 3.0, dtype=torch.bfloat16)
    assert torch.equal(c.marks.cpu(), landmarks64(pool, 32, first, old))
    c.landmarks(first=_i32([-7, -1, 0, 0]))
    assert torch.equal(c.marks.cpu(), landmarks64(pool, 32, None, old))


def test_lists_of_a_caller():
    """Any ascending lists: blocks past a token's own, empty ones, own block left out."""
    pool = make("bf16", [500, 300], 2, 16, seed=9)
    tokens = [(0, 499), (0, 400), (1, 299), (0, 398), (1, 10)]
    req, pos = [t[0] for t in tokens], [t[1] for t in tokens]
    idx = torch.tensor([[[0, 3, 7, -1], [-1, -1, -1, -1]], [[2, 3, 12, 15], [12, 13, 14, 15]],
                        [[9, 10, 11, 1 << 30], [0, -1, -1, -1]], [[3, 12, -1, -1], [0, 1, 2, 3]],
                        [[0, 1, 2, 3], [5, 6, 7, 8]]], dtype=torch.int32)
    q = torch.randn((5, 8, D), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    c = Call(pool, 4, 32, 4, 5)
    c.idx.copy_(idx)
    c.attend(_i32(req), _i32(pos), q.to(DEV))
    out, lse, tol = attend64(pool, 32, req, pos, q, idx)
    none = lse == -math.inf
    assert none.any() and torch.all(c.out.cpu()[none] == 0)
    assert torch.equal(c.lse.cpu() == -math.inf, none)
    assert torch.all((c.out.cpu().double() - out).abs().amax(-1) <= tol)


@pytest.mark.parametrize("kind,new,Hkv,G", [("e4m3", 30, 2, 4), ("bf16", 800, 2, 16),
                                             ("bf16", 1030, 2, 16)])
def test_a_block_named_twice_counts_once(kind, new, Hkv, G):
    """The same block twice in a list, blocks past the token's own after them."""
    n, block = max(900, new + 70), 64
    pool = make(kind, [n], Hkv, 16, seed=new)
    pos = torch.arange(n - new, n, dtype=torch.int32)
    own = pos // block
    once = torch.full((new, Hkv, 6), -1, dtype=torch.int32)
    once[:, :, 0], once[:, :, 1] = 0, own[:, None]
    twice = torch.full((new, Hkv, 6), 1 << 28, dtype=torch.int32)
    twice[:, :, :3], twice[:, :, 3:5] = 0, own[:, None, None]
    q = torch.randn((new, G * Hkv, D), generator=torch.Generator().manual_seed(1))
    q = q.to(torch.bfloat16).to(DEV)
    got = []
    for idx in (once, twice):
        c = Call(pool, G, block, 6, new)
        c.idx.copy_(idx)
        c.attend(torch.zeros_like(pos).to(DEV), pos.to(DEV), q)
        got += [c.out, c.lse]
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[3])
    assert torch.isfinite(got[0]).all()


def test_all_blocks_kept_is_the_whole_attention():
    """With every block kept a token gets what the decode attention gives it."""
    lens = [300, 450]
    pool = make("e2m1", lens, 2, 16, seed=6, max_ctx=450)
    T, G = 4, 4
    q = torch.randn((2, T, 2 * G, D), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    want, wl, tol = pool.attention(q, T)
    tokens = ragged_tokens(lens, T)
    c = Call(pool, G, 32, 15, 2 * T)
    r, p = _i32([t[0] for t in tokens]), _i32([t[1] for t in tokens])
    qd = q.view(2 * T, 2 * G, D).to(DEV)
    c.landmarks()
    c.select(r, p, qd)
    c.attend(r, p, qd)
    assert torch.all((c.out.cpu().double().view_as(want) - want).abs().amax(-1) <= tol)


@pytest.mark.parametrize("new,G", [(1, 4), (200, 4)])
def test_captured_and_replayed_and_on_another_stream(new, G):
    """One capture of the three calls replayed over changing tokens, with eager
    calls between the replays and on another stream; the same bits every time."""
    lens = [900, 700, 650]
    pool = make("e2m1", lens, 2, 32, seed=12, max_ctx=1000)
    tokens = ragged_tokens(lens, new)
    n = len(tokens)
    c, e = Call(pool, G, 64, 5, n), Call(pool, G, 64, 5, n)
    r, p = _i32([t[0] for t in tokens]), _i32([t[1] for t in tokens])
    first = pool.ctx - new
    q = torch.randn((n, G * 2, D), device=DEV).to(torch.bfloat16)
    g = torch.Generator(device=DEV).manual_seed(7)

    def run(x, stream=None):
        x.landmarks(first=first, stream=stream)
        x.select(r, p, q, stream=stream)
        x.attend(r, p, q, stream=stream)

    for x in (c, e):
        x.landmarks()
    run(c)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(c)
    side = torch.cuda.Stream()
    for i in range(4):
        q.copy_(torch.randn(q.shape, generator=g, device=DEV))
        p.copy_(torch.where(p > 64 * i, p - 7, p))
        graph.replay()
        torch.cuda.synchronize()
        run(e, side if i % 2 else None)
        torch.cuda.synchronize()
        for a, b in ((c.marks, e.marks), (c.idx, e.idx), (c.out, e.out), (c.lse, e.lse)):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("Hkv,G,block,k,page,order,new", [
    (2, 16, 64, 6, 16, "pairs", 400), (8, 4, 32, 17, 64, "heads", 350),
    (16, 1, 128, 3, 16, "rows", 700), (4, 8, 256, 2, 32, "heads", 350)])
def test_many_tokens_of_a_bf16_cache(Hkv, G, block, k, page, order, new):
    """Four tiles a workgroup: chunks of three requests, holes, padding and a
    request's tokens apart from each other; every seventh token is compared."""
    _log("many", Hkv, G, block, k, page, order, new)
    lens = [900, 640, 1001]
    pool = make("bf16", lens, Hkv, page, seed=G, order=order, holes=[(0, 1), (2, 3), (1, 0)],
                max_ctx=1010)
    tokens = ragged_tokens(lens, new)
    tokens = tokens[:100] + [(0, -1), (3, 5), (0, 0), (2, 31)] + tokens[100:-5] + [(1, 500)]
    req, pos = [t[0] for t in tokens], [t[1] for t in tokens]
    g = torch.Generator().manual_seed(new)
    q = torch.randn((len(tokens), G * Hkv, D), generator=g).to(torch.bfloat16)
    c = Call(pool, G, block, k, len(tokens))
    r, p, qd = _i32(req), _i32(pos), q.to(DEV)
    c.landmarks()
    c.select(r, p, qd)
    idx = c.idx.cpu()
    c.attend(r, p, qd)
    some = sorted({*range(0, len(tokens), 7), 100, 101, 102, 103, len(tokens) - 1})
    rq, ps = [req[i] for i in some], [pos[i] for i in some]
    assert torch.equal(idx[some], select64(pool, block, k, rq, ps, q[some], c.marks.cpu()))
    out, lse, tol = attend64(pool, block, rq, ps, q[some], idx[some])
    got, gl = c.out.cpu().double()[some], c.lse.cpu().double()[some]
    none = lse == -math.inf
    assert none.any() and torch.all(got[none] == 0) and torch.all(gl[none] == -math.inf)
    err = (got - out).abs().amax(-1)
    assert torch.all(err <= tol), float((err / tol.clamp(min=1e-30)).max())
    assert torch.all(((gl - lse).abs() <= tol + 2.0 ** -22 * lse.abs() + 1e-6)[~none])


@pytest.mark.parametrize("kind,new,Hkv,G", [
    ("bf16", 40, 2, 4), ("e4m3", 40, 2, 2), ("e2m1", 40, 2, 8), ("bf16", 3, 2, 1),
    ("e2m1", 3, 2, 4), ("bf16", 780, 2, 16), ("bf16", 1030, 2, 16), ("bf16", 1030, 8, 4)])
def test_rows_that_are_no_numbers_reach_only_who_sees_them(kind, new, Hkv, G):
    """NaN and infinite rows of K and V, seen by some tokens of a tile and not by
    others (another block, a later position): the others' outputs are as without."""
    _log("no numbers", kind, new, Hkv, G)
    n, block, k = max(1000, new + 200), 32, 4
    pool = make(kind, [n], Hkv, 16, seed=new)
    g = torch.Generator().manual_seed(5)
    pos = list(range(n - new, n))
    own = torch.tensor(pos) // block
    idx = torch.full((new, Hkv, k), -1, dtype=torch.int32)
    for t in range(new):
        for h in range(Hkv):
            few = sorted(torch.randperm(6, generator=g)[:k - 1].tolist())
            idx[t, h] = torch.tensor(few + [int(own[t])])
    poison(pool, 0, 0, 2 * block + 7, "v")
    poison(pool, 0, Hkv - 1, 4 * block, "v", math.inf)
    poison(pool, 0, Hkv - 1, 5 * block + 31, "k")
    poison(pool, 0, 0, n - 1, "v")          # of the last token's own block
    poison(pool, 0, Hkv - 1, n - 2, "k", -math.inf if kind == "bf16" else 0)
    q = torch.randn((new, G * Hkv, D), generator=g).to(torch.bfloat16)
    c = Call(pool, G, block, k, new)
    c.idx.copy_(idx)
    c.attend(_i32([0] * new), _i32(pos), q.to(DEV))
    some = sorted({*range(0, new, max(1, new // 60)), *range(max(0, new - 20), new)})
    out, lse, tol = attend64(pool, block, [0] * len(some), [pos[i] for i in some], q[some],
                             idx[some])
    got = c.out.cpu().double()[some]
    good = torch.isfinite(out)
    assert good.any() and not good.all()
    assert torch.equal(torch.isfinite(got), good)
    rows = good.all(-1)
    assert rows.any()
    err = (got - out)[rows].abs().amax(-1)
    assert torch.all(err <= tol[rows])


def test_many_tokens_captured_and_replayed():
    """Staged blocks of four tiles in a graph: changing queries and positions, eager
    calls on another stream between the replays."""
    n, Hkv, G = 1030, 2, 16
    pool = make("bf16", [1200], Hkv, 16, seed=4)
    c, e = Call(pool, G, 64, 5, n), Call(pool, G, 64, 5, n)
    p = torch.arange(1200 - n, 1200, dtype=torch.int32, device=DEV)
    r = torch.zeros_like(p)
    q = torch.randn((n, G * Hkv, D), device=DEV).to(torch.bfloat16)

    def run(x, stream=None):
        x.select(r, p, q, stream=stream)
        x.attend(r, p, q, stream=stream)

    for x in (c, e):
        x.landmarks()
        run(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(c)
    side = torch.cuda.Stream()
    for i in range(4):
        q.copy_(torch.randn(q.shape, device=DEV))
        p.sub_(i)
        graph.replay()
        torch.cuda.synchronize()
        run(e, side if i % 2 else None)
        torch.cuda.synchronize()
        assert torch.equal(c.idx, e.idx) and torch.equal(c.out, e.out) and torch.equal(c.lse, e.lse)


def test_debug_mode_names_bad_tokens():
    pool = make("bf16", [100, 50], 1, 16, seed=1, holes=[(1, 3)])
    c = Call(pool, 1, 32, 2, 2)
    q = torch.zeros((2, 1, D), dtype=torch.bfloat16, device=DEV)
    c.landmarks()
    ckv.set_debug(True)
    try:
        c.select(_i32([0, 1]), _i32([99, 49]), q)   # a token may lack its page
        c.attend(_i32([0, 1]), _i32([99, -1]), q)
        for req, pos, text in (([0, 2], [0, 0], r"requests\[1\]"), ([0, 1], [100, 0],
                                                                     r"positions\[0\]")):
            with pytest.raises(ckv.CkvError, match=text):
                c.select(_i32(req), _i32(pos), q)
            with pytest.raises(ckv.CkvError, match=text):
                c.attend(_i32(req), _i32(pos), q)
    finally:
        ckv.set_debug(False)


def test_kernels_that_run():
    """A few tokens are cut into pieces and joined, many are not."""
    pool = make("bf16", [2000], 1, 16, seed=1)
    for n, merge in ((1, 1), (1900, 0)):
        c = Call(pool, 16, 32, 32, n)
        p = torch.arange(2000 - n, 2000, dtype=torch.int32, device=DEV)
        q = torch.randn((n, 16, D), device=DEV).to(torch.bfloat16)
        req = torch.zeros_like(p)
        ckv.profile_begin()
        c.landmarks()
        c.select(req, p, q)
        c.attend(req, p, q)
        ran = ckv.profile_end()
        assert {k: v[0] for k, v in ran.items()} == {
            "block_marks": 1, "block_score": 1, "block_select": 1, "block_attn": 1,
            **({"block_merge": 1} if merge else {})}
