"""Attention with changed scores (cap, slopes over positions) and its log-sum-exp against the 64-bit definition."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as K
from paper_2506_14158_amd import binding as B
from paper_2506_14158_amd.verify import TreeVerifier

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CODE = {"f32": B.S4C_F32, "bf16": B.S4C_BF16, "f16": B.S4C_F16}
HALF_STEP = {t: torch.finfo(DT[t]).eps / 2 for t in DT}


def f64(t):
    return t.detach().double().cpu().numpy()


class Case:
    def __init__(self, seed, B_, N, Hq, Hkv, D, dtype, lengths, S_cap, page=0, chain=False, q_std=2.0):
        g = torch.Generator().manual_seed(seed)
        r = np.random.default_rng(seed)
        f = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(DT[dtype]).cuda()
        self.shape = B.AttnShape(B_, Hq, Hkv, D, N, S_cap, CODE[dtype])
        self.dtype, self.page = dtype, page
        self.q, self.kt, self.vt = f(B_, N, Hq, D, std=q_std), f(B_, N, Hkv, D), f(B_, N, Hkv, D)
        self.table = None
        if page:
            blocks = S_cap // page
            self.kc, self.vc = f(B_ * blocks + 1, Hkv, page, D), f(B_ * blocks + 1, Hkv, page, D)
            self.table = torch.from_numpy(r.permutation(B_ * blocks + 1)[:B_ * blocks].reshape(B_, blocks).astype(np.int32)).cuda()
        else:
            self.kc, self.vc = f(B_, Hkv, S_cap, D), f(B_, Hkv, S_cap, D)
        parent = np.full((B_, N), -1, dtype=np.int32)
        for b in range(B_):
            for i in range(1, N):
                parent[b, i] = i - 1 if chain else r.integers(max(0, i - 7), i)
        self.parent = torch.from_numpy(parent).cuda()
        self.len = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.slopes = torch.tensor([2.0 ** (-6.0 * (h + 1) / Hq) for h in range(Hq)], dtype=torch.float32, device="cuda")
        # positions of a cache that rows were evicted from: any order, far from zero
        self.pos = torch.from_numpy(np.stack([[r.permutation(3 * S_cap)[:S_cap] for _ in range(Hkv)] for _ in range(B_)]).astype(np.int32)).cuda()
        self.pos += 1 << 30
        self.root = torch.full((B_,), (1 << 30) + 3 * S_cap, dtype=torch.int32, device="cuda")
        self.out = torch.full_like(self.q, 7.0)
        self.lse = torch.full((B_, N, Hq), 7.0, device="cuda")
        self.status = torch.full((B_,), 9, dtype=torch.int32, device="cuda")

    def score(self, cap, bias):
        return B.Score(cap, self.slopes if bias != "none" else None, *((self.pos, self.root) if bias == "kept" else (None, None)))

    def call(self, score, max_len=None, scale=0.0, lse=True, ws=None):
        m = int(self.len.clamp(min=0).max()) if max_len is None else max_len
        ws = B.alloc_workspace(B.s4c_tree_attn_workspace_size(self.shape, m)) if ws is None else ws
        lse = self.lse if lse else None
        if self.page:
            B.s4c_tree_attn_scored_paged(self.q, self.kt, self.vt, self.kc, self.vc, self.table, self.len, self.parent, m, score, self.out, lse,
                                         scale, self.status, ws)
        else:
            B.s4c_tree_attn_scored(self.q, self.kt, self.vt, self.kc, self.vc, self.len, self.parent, m, score, self.out, lse, scale, self.status, ws)
        torch.cuda.synchronize()

    def caches(self):
        if not self.page:
            return f64(self.kc), f64(self.vc)
        t = self.table.cpu().numpy()
        return K.gather_pages(f64(self.kc), t), K.gather_pages(f64(self.vc), t)

    def want(self, score, scale=0.0):
        kc, vc = self.caches()
        n = lambda t: None if t is None else t.cpu().numpy()
        slopes = None if score.slopes is None else f64(score.slopes)
        return K.tree_attn_scored(f64(self.q), f64(self.kt), f64(self.vt), kc, vc, n(self.len), n(self.parent), scale, score.cap, slopes,
                                  n(score.key_pos), n(score.root_pos))

    def check(self, score, scale=0.0, rows=slice(None)):
        """Per value, to first order.  A score is off by its D fp32 additions (2^-24 of sum |q k| each) and by at most 12 roundings of half a
        step of its own size (the conversion to log2 units, the cap's seven operations, the bias, the difference to the reference) and, beyond the
        fit, by 2^-22 of the cap; the log-sum-exp by the mean of that under the softmax, the n + 40 additions of its sum and a few
        roundings; the output by the same weighted with |v| + |out|, by half a step of every probability where those are rounded (16-bit data
        of head size 128), 2^-21 for exponentials and the merge, and its own rounding."""
        out, lse, mean, mean_s, size, mass = self.want(score, scale)
        D, n = self.shape.D, float(self.len.max()) + self.shape.N
        hs, u = HALF_STEP[self.dtype], 2.0 ** -24
        every = u * (D * mass + 6 * score.cap) + u * (n + 40)
        p = every + 2.0 ** -21 + (hs if D == 128 and self.dtype != "f32" else 0.0)
        got, got_lse = f64(self.out), f64(self.lse)
        err = np.abs(got - out)[rows]
        tol = p[..., None] * (mean + np.abs(out)) + 12 * u * (mean_s + size[..., None] * np.abs(out))
        tol = (1.01 * (tol + hs * (np.abs(out) + tol)) + 2.0 ** -30)[rows]
        assert (err <= tol).all(), (err.max(), (err / tol).max())
        err = np.abs(got_lse - lse)[rows]
        tol = (1.01 * (every + 12 * u * size + 2.0 ** -22 * (np.abs(lse) + 16)))[rows]
        assert (err <= tol).all(), (err.max(), (err / tol).max())
        # all in all, roundings do not add up: a few half steps (and fp32's errors) in the 2-norm
        rel = np.linalg.norm((got - out)[rows]) / np.linalg.norm(out[rows])
        assert rel <= (4 * hs if self.dtype != "f32" else 1e-5), rel


SHAPES = {
    # name: B, N, Hq, Hkv, D, lengths, S_cap, page
    "one token, short": (3, 1, 4, 4, 64, (0, 1, 33), 64, 0),
    "one token, grouped": (2, 1, 16, 2, 128, (700, 513), 768, 0),
    "odd tree": (2, 13, 6, 2, 128, (100, 37), 128, 0),
    "empty prefixes": (2, 64, 4, 2, 64, (0, 0), 64, 0),
    "32 rows, many units": (5, 8, 32, 8, 64, (300, 1, 64, 299, 150), 320, 0),
    "64 rows": (1, 32, 8, 4, 128, (1500,), 1536, 0),
    "over 64 rows": (2, 40, 8, 4, 128, (321, 255), 384, 0),
    "over 128 rows": (1, 128, 8, 4, 64, (513,), 576, 0),
    "over 256 rows": (1, 70, 8, 2, 128, (450,), 512, 0),
    "paged, ragged": (3, 21, 8, 2, 128, (129, 640, 64), 640, 64),
    "paged, head size 64": (2, 5, 8, 8, 64, (255, 130), 256, 128),
    "long, few units": (1, 3, 2, 1, 128, (9001,), 9216, 0),
}
SCORES = [(0.0, "none"), (30.0, "none"), (2.0, "none"), (0.0, "rows"), (5.0, "rows"), (0.0, "kept"), (20.0, "kept")]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("name", SHAPES)
def test_against_the_definition(name, dtype):
    B_, N, Hq, Hkv, D, lengths, S_cap, page = SHAPES[name]
    c = Case(sum(map(ord, name)), B_, N, Hq, Hkv, D, dtype, lengths, S_cap, page)
    large = N * Hq * sum(lengths) > 200000
    for cap, bias in SCORES[1::3] + SCORES[:1] if large else SCORES:
        c.out.fill_(7.0)
        c.lse.fill_(7.0)
        c.call(c.score(cap, bias))
        assert not c.status.any()
        c.check(c.score(cap, bias))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_far_beyond_the_cap(dtype):
    """|x / cap| from 0 to 60 in one wave: tanh on both of its ways, and saturated."""
    c = Case(5, 1, 9, 4, 2, 64, dtype, (200,), 256, q_std=8.0)
    for cap in (0.25, 1.0, 12.0):
        c.call(c.score(cap, "none"))
        c.check(c.score(cap, "none"))


@pytest.mark.parametrize("N", [7, 80])
def test_caps_at_the_ends_of_their_range(N):
    """A cap so wide that it does nothing, one so narrow that only signs are left, and scores that are all zero."""
    c = Case(14, 1, N, 4, 2, 128, "bf16", (200,), 256)
    for cap in (1e20, 1e5, 1e-3, 1e-20):
        c.call(c.score(cap, "rows"))
        c.check(c.score(cap, "rows"))
        c.call(c.score(cap, "none"))
        c.check(c.score(cap, "none"))
    c.q.zero_()
    for cap in (1e20, 30.0, 1e-20):
        c.call(c.score(cap, "none"))
        c.check(c.score(cap, "none"))


@pytest.mark.parametrize("N,bias", [(7, "none"), (80, "none"), (80, "rows")])
def test_capped_scores_whose_squares_are_not_finite(N, bias):
    """Scores of 2^69 k, k = 0 .. 4, and one of 2^72, the cap; every other row's weight is 0 and the output that one row's value."""
    c = Case(15, 1, N, 4, 2, 128, "bf16", (256,), 256)
    c.q.zero_()
    c.q[..., 0] = 2.0 ** 35
    c.kt.zero_()
    c.kc.zero_()
    c.kc[:, :, :, 0] = 2.0 ** 34 * (torch.arange(256, device="cuda") % 5).to(torch.bfloat16)
    c.kc[:, :, 100, 0] = 2.0 ** 37
    c.call(c.score(2.0 ** 72, bias), scale=1.0)
    c.check(c.score(2.0 ** 72, bias), scale=1.0)
    assert torch.equal(c.out, c.vc[:, None, :, 100].repeat_interleave(2, 2).expand(1, N, 4, 128))


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    r = np.random.default_rng([seed, 5])
    D, G, Hkv, B_ = int(r.choice([64, 128])), int(r.choice([1, 2, 3, 4, 8])), int(r.choice([1, 2, 3])), int(r.integers(1, 4))
    N = int(r.choice([1, 2, r.integers(3, 129)]))
    page = int(r.choice([0, 0, 64, 128]))
    top = int(np.exp(r.uniform(np.log(4), np.log(1200))))
    while N * G * Hkv * B_ * top > 400000:
        top //= 2
    lengths = [int(r.integers(0, top + 1)) for _ in range(B_)]
    S_cap = -(-max(top, 1) // (page or 8)) * (page or 8)
    c = Case(seed + 100, B_, N, Hkv * G, Hkv, D, str(r.choice(["bf16", "f16", "f32"])), lengths, S_cap, page, chain=bool(r.random() < 0.3))
    for _ in range(2):
        s = c.score(float(r.choice([0.0, 1.0, 10.0, 40.0])), str(r.choice(["none", "rows", "kept"])))
        c.out.fill_(7.0)
        c.lse.fill_(7.0)
        c.call(s, max_len=int(r.integers(max(lengths), S_cap + 1)))
        c.check(s)


def test_another_scale_and_a_longer_bound():
    """`scale` is the caller's; max_cache_len only sizes the launch."""
    c = Case(6, 2, 10, 4, 2, 128, "f16", (90, 300), 1024)
    s = c.score(10.0, "rows")
    c.call(s, max_len=1024, scale=0.03)
    c.check(s, scale=0.03)


def test_balanced_shares_have_their_lse_too():
    """Ragged units laid end to end: parts merged by a launch of their own, whole units beside them."""
    lengths = [2000 + 97 * i for i in range(13)]
    c = Case(7, 13, 20, 8, 8, 64, "f16", lengths, 4096)
    s = c.score(15.0, "kept")
    c.call(s)
    rows = (slice(None, None, 5), slice(None, None, 7), slice(None))
    c.check(s, rows=rows)


def test_without_changes_it_is_the_plain_attention():
    """The same probabilities up to the rounding of a score (a product with the scale instead of a fused one)."""
    for dtype, N in (("bf16", 60), ("f16", 7), ("f32", 20)):
        c = Case(8, 2, N, 8, 4, 128, dtype, (777, 512), 1024)
        c.call(B.PLAIN_SCORE)
        plain = torch.empty_like(c.out)
        ws = B.alloc_workspace(B.s4c_tree_attn_workspace_size(c.shape, 777))
        B.s4c_tree_attn(c.q, c.kt, c.vt, c.kc, c.vc, c.len, c.parent, 777, plain, 0.0, c.status, ws)
        hs = HALF_STEP[dtype]
        assert (plain.double() - c.out.double()).norm() <= (2 * hs if dtype != "f32" else 1e-6) * plain.double().norm()
        # and without lse, with no array for it
        first = c.out.clone()
        c.call(B.PLAIN_SCORE, lse=False)
        assert torch.equal(first, c.out)


@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("N", [5, 90])
def test_flagged_sequences(page, N):
    """A bad tree, lengths out of range, a bad page: status, zero output, lse +infinity; the others are not touched by it."""
    c = Case(9, 4, N, 4, 2, 128, "bf16", (200, 100, 130, 64), 256, page)
    s = c.score(20.0, "rows")
    c.call(s, max_len=200)
    good = (c.out.clone(), c.lse.clone())
    c.parent[1, 3] = 3
    c.len[2] = 201
    if page:
        c.table[3, 0] = c.kc.shape[0]
    c.call(s, max_len=200)
    assert c.status.tolist() == [0, B.S4C_SEQ_BAD_TREE, B.S4C_SEQ_BAD_LEN, B.S4C_SEQ_BAD_LEN if page else 0]
    bad = [1, 2] + ([3] if page else [])
    for b in range(4):
        if b in bad:
            assert not c.out[b].any() and (c.lse[b] == float("inf")).all()
        else:
            assert torch.equal(c.out[b], good[0][b]) and torch.equal(c.lse[b], good[1][b])


def test_replayed_and_on_another_stream():
    """A captured call replayed with other lengths in between eager ones, and a call on a side stream: bit-equal to the eager results."""
    c = Case(10, 3, 17, 8, 4, 64, "bf16", (900, 1400, 33), 1536)
    s = c.score(25.0, "kept")
    ws = B.alloc_workspace(B.s4c_tree_attn_workspace_size(c.shape, 1500))
    lengths = [(900, 1400, 33), (1500, 0, 64), (1, 1023, 1499)]
    want = []
    for n in lengths:
        c.len.copy_(torch.tensor(n, dtype=torch.int32))
        c.call(s, max_len=1500, ws=ws)
        want.append((c.out.clone(), c.lse.clone()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.call(s, max_len=1500, ws=ws)
    assert torch.equal(c.out, want[-1][0]) and torch.equal(c.lse, want[-1][1])
    graph = torch.cuda.CUDAGraph()
    run = lambda: B.s4c_tree_attn_scored(c.q, c.kt, c.vt, c.kc, c.vc, c.len, c.parent, 1500, s, c.out, c.lse, 0.0, c.status, ws)
    with torch.cuda.graph(graph):
        run()
    for i in (0, 1, 2, 0, 2, 1):
        c.len.copy_(torch.tensor(lengths[i], dtype=torch.int32))
        c.out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, want[i][0]) and torch.equal(c.lse, want[i][1])
        run()
        assert torch.equal(c.out, want[i][0])


def test_two_calls_at_once():
    """Two streams, a workspace each: both as if alone."""
    cs = [Case(20 + i, 2, 33, 8, 4, 128, "bf16", (1200, 700), 1280) for i in range(2)]
    want = []
    for c in cs:
        c.call(c.score(30.0, "rows"))
        want.append(c.out.clone())
    ws = [B.alloc_workspace(B.s4c_tree_attn_workspace_size(c.shape, 1200)) for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, st, w in zip(cs, streams, ws):
            with torch.cuda.stream(st):
                B.s4c_tree_attn_scored(c.q, c.kt, c.vt, c.kc, c.vc, c.len, c.parent, 1200, c.score(30.0, "rows"), c.out, c.lse, 0.0, c.status, w)
    torch.cuda.synchronize()
    for c, w in zip(cs, want):
        assert torch.equal(c.out, w)


def test_positions_beyond_32_bit_offsets():
    """A cache of more than 2^31 elements: rows and positions of its last sequence."""
    S_cap, n = 1 << 23, 500
    pool = torch.zeros(3, 1, S_cap, 128, dtype=torch.bfloat16, device="cuda")
    c = Case(11, 3, 4, 2, 1, 128, "bf16", (3, 5, n), 512)
    pos = torch.zeros(3, 1, S_cap, dtype=torch.int32, device="cuda")
    small = (c.kc, c.vc)
    for b in range(3):
        pool[b, :, :512] = c.kc[b]
        pos[b, :, :512] = c.pos[b]
    c.kc = pool
    c.vc = pool.clone()
    for b in range(3):
        c.vc[b, :, :512] = small[1][b]
    c.shape.S_cap = S_cap
    s = B.Score(20.0, c.slopes, pos, c.root)
    c.call(s)
    c.kc, c.vc = small
    c.check(c.score(20.0, "kept"))


def test_refusals():
    c = Case(12, 2, 6, 4, 2, 64, "bf16", (50, 20), 64)
    ws = B.alloc_workspace(max(256, B.s4c_tree_attn_workspace_size(c.shape, 50)))

    def call(score=B.PLAIN_SCORE, q=c.q, out=c.out, lse=c.lse, length=c.len, status=c.status, m=50):
        B.s4c_tree_attn_scored(q, c.kt, c.vt, c.kc, c.vc, length, c.parent, m, score, out, lse, 0.0, status, ws)
    call()
    for cap in (-1.0, float("nan"), float("inf"), 3.3e38, 1e-40):
        with pytest.raises(B.S4CError) as e:
            call(B.Score(cap))
        assert e.value.code == -2
    with pytest.raises(B.S4CError) as e:
        call(B.Score(0.0, c.slopes, c.pos))                     # positions of the keys, none of the root
    assert e.value.code == -1
    for bad in (B.Score(0.0, c.slopes[:3].contiguous()), B.Score(0.0, c.slopes.double()), B.Score(0.0, c.slopes, c.pos.long(), c.root),
                B.Score(0.0, c.slopes, c.pos[:, :, :50].contiguous(), c.root), B.Score(0.0, c.slopes, c.pos, c.root[:1])):
        with pytest.raises(TypeError):
            call(bad)
    with pytest.raises(TypeError):
        call(lse=c.lse.half())
    with pytest.raises(TypeError):
        call(status=c.status[:1])
    with pytest.raises(TypeError):
        call(length=c.len[:1])
    with pytest.raises(TypeError):
        call(out=c.out.float())
    with pytest.raises(ValueError):
        call(B.Score(0.0, torch.ones(8, device="cuda")[::2]))   # not contiguous
    with pytest.raises(ValueError):
        call(B.Score(0.0, torch.ones(4)))                       # not on the device
    with pytest.raises(B.S4CError):
        call(m=65)
    with pytest.raises(TypeError):
        B.s4c_tree_attn_scored_paged(c.q, c.kt, c.vt, c.kc, c.vc, None, c.len, c.parent, 50, B.PLAIN_SCORE, c.out)


def test_verifier_attends_with_a_score():
    c = Case(13, 2, 12, 4, 2, 64, "f16", (100, 64), 192)
    v = TreeVerifier(2, 12, 4, 2, 64, 192, 100, torch.float16, 12, 160)
    s = c.score(8.0, "rows")
    c.call(s, max_len=160)
    v.tree_attn_scored(c.q, c.kt, c.vt, c.kc, c.vc, c.len, c.parent, s)
    assert torch.equal(v.out, c.out) and torch.equal(v.lse, c.lse)
