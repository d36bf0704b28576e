"""Latent cache and attention on the GPU against a float64 reference (tests/latent_ref.py):
stores with norm, rotation and 8-bit latents, read-back, both attention entry points and
both forms, at the sizes and masks where they can go wrong."""

import math

import numpy as np
import pytest
import torch

import helpers
import latent_ref as ref
from paper_2609_32278_amd import kvx

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16


class Setup:
    """A pool whose every slot holds NaN, a shuffled page table and the cached rows of a batch."""

    def __init__(self, P, E, lat, fp8, seed=0, poison=True, extra_pages=5):
        g = torch.Generator(DEV).manual_seed(seed)
        self.P, self.E, self.lat, self.fp8, self.g = list(P), list(E), lat, fp8, g
        need = [-(-(p + e) // 16) for p, e in zip(P, E)]
        self.indptr = np.concatenate([[0], np.cumsum(need)]).astype(np.int32)
        self.num_pages = int(self.indptr[-1]) + extra_pages
        self.ids = torch.randperm(self.num_pages, device=DEV, generator=g).to(torch.int32)
        self.pages = self.ids[: int(self.indptr[-1])].contiguous()
        self.pool = kvx.latent_pool_create(self.num_pages, 16, lat, 64, kvx.KVX_LATENT_FP8 if fp8 else kvx.KVX_LATENT_BF16)
        if poison:
            n = self.num_pages * 16
            self.store_all(torch.full((n, lat + 64), float("nan"), dtype=BF16, device=DEV))
        self.batch = kvx.Batch(P, E, self.indptr, self.pages)
        self.T = self.batch.total_extend

    def store_all(self, rows):
        n = self.num_pages
        kvx.store_latent(self.pool, kvx.Batch([0], [n * 16], [0, n], self.ids), rows)

    def load_all(self):
        n = self.num_pages
        out = torch.empty(n * 16, self.lat + 64, dtype=BF16, device=DEV)
        kvx.load_latent(self.pool, kvx.Batch([0], [n * 16], [0, n], self.ids), out)
        return out.view(n, 16, -1)

    def normal(self, *shape, scale=1.0):
        return torch.randn(shape, device=DEV, generator=self.g, dtype=BF16) * scale

    def fill(self, scale=1.0, rows=None):
        """Cache the whole sequences; returns the rows the pool then stands for (float64)."""
        lens = [p + e for p, e in zip(self.P, self.E)]
        rows = self.normal(sum(lens), self.lat + 64, scale=scale) if rows is None else rows
        kvx.store_latent(self.pool, kvx.Batch([0] * len(lens), lens, self.indptr, self.pages), rows)
        x = ref.f64(rows)
        if self.fp8:
            x[:, : self.lat] = ref.quantised(x[:, : self.lat])
        cuts = np.cumsum([0] + lens)
        return [x[cuts[i]:cuts[i + 1]] for i in range(len(lens))]

    def close(self):
        torch.cuda.synchronize()
        kvx.latent_pool_destroy(self.pool)


@pytest.fixture
def setup():
    made = []

    def make(*a, **k):
        made.append(Setup(*a, **k))
        return made[-1]

    yield make
    for s in made:
        s.close()


# ------------------------------------------------------------------- store and load

BATCHES = [
    ([0], [1]),
    ([5], [11]),                               # ends with the page
    ([15], [2]),                               # across a page border
    ([0, 37, 16, 100], [40, 0, 16, 3]),        # an empty request, whole pages, unaligned ends
    (list(range(0, 130)), [1 + i % 3 for i in range(130)]),  # more requests than the arguments hold
]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lat", [256, 512])
@pytest.mark.parametrize("P,E", BATCHES)
def test_store_then_load(setup, P, E, lat, fp8):
    s = setup(P, E, lat, fp8)
    wide = s.normal(s.T, lat + 64 + 24, scale=3.0)  # rows inside wider rows
    wide[:, : lat] *= torch.exp2(torch.randint(-20, 20, (s.T, lat), device=DEV, generator=s.g).float()).to(BF16)
    wide[0, :64] = 0.0
    rows = wide[:, 8:8 + lat + 64] if lat % 16 == 0 else wide
    before = s.load_all()
    kvx.store_latent(s.pool, s.batch, rows)
    out = torch.full((s.T + 2, lat + 64 + 16), 7.0, dtype=BF16, device=DEV)
    kvx.load_latent(s.pool, s.batch, out[1:1 + s.T, 8:8 + lat + 64])
    want = ref.f64(rows)
    if fp8:
        want[:, :lat] = ref.quantised(want[:, :lat])
    assert (ref.f64(out[1:1 + s.T, 8:8 + lat + 64]) == want).all()
    # rows before and behind, and columns beside, are kept
    assert (out[0] == 7).all() and (out[-1] == 7).all() and (out[:, :8] == 7).all() and (out[:, lat + 72:] == 7).all()
    # so are all slots that the batch does not own
    after = s.load_all()
    touched = torch.zeros(s.num_pages, 16, dtype=torch.bool, device=DEV)
    where = {int(p): i for i, p in enumerate(s.ids)}
    for r, (p, e) in enumerate(zip(P, E)):
        for t in range(p, p + e):
            touched[where[int(s.pages[int(s.indptr[r]) + t // 16])], t % 16] = True
    assert torch.equal(before.view(torch.int16)[~touched], after.view(torch.int16)[~touched])


def test_store_special_values(setup):
    """Infinities saturate an 8-bit group, NaN stays with its value, tiny groups reach the
    smallest scale, the largest bf16 value stays finite."""
    for fp8 in (False, True):
        s = setup([0], [4], 256, fp8, poison=False)
        x = torch.zeros(4, 320, dtype=BF16, device=DEV)
        x[0, 3], x[0, 70], x[0, 130], x[0, 300] = math.inf, -math.inf, math.nan, math.nan
        x[0, 131] = 2.0
        x[1, :64] = 2.0 ** -126
        x[1, 64:128] = 2.0 ** -133
        x[2, :4] = torch.tensor([torch.finfo(BF16).max, -torch.finfo(BF16).max, 1.0, 2.0 ** 118])
        kvx.store_latent(s.pool, s.batch, x)
        out = torch.empty_like(x)
        kvx.load_latent(s.pool, s.batch, out)
        if not fp8:
            assert torch.equal(out.view(torch.int16), x.view(torch.int16))
            continue
        top = 448 * 2.0 ** 119
        assert out[0, 3] == top and out[0, 70] == -top and out[0, 131] == 2.0
        assert out[0, 130].isnan() and out[0, 300].isnan()
        assert (out[1, :64] == 2.0 ** -126).all()
        assert (out[1, 64:128] == 0).all()  # below half of the smallest step, 2^-9 * 2^-117
        assert out[2, 0] == top and out[2, 1] == -top and out[2, 3] == 2.0 ** 118


@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("lat,hd,heads,fp8,in_place", [
    (512, 128, 3, False, False), (512, 128, 16, True, True), (256, 64, 1, True, False), (256, 0, 5, False, False),
    (512, 72, 37, False, True), (256, 64, 0, False, False)])
def test_store_rope(setup, style, lat, hd, heads, fp8, in_place):
    P, E = [0, 250, 16, 1000], [17, 1, 0, 30]
    s = setup(P, E, lat, fp8)
    kv = s.normal(s.T, lat + 64, scale=2.0)
    norm = 1.0 + s.normal(lat, scale=0.3)
    q = s.normal(s.T, max(heads, 1), hd + 64)
    given = q.clone()
    q_out = q if in_place else torch.full_like(q, 9.0)
    theta = 1e4 if style else 1e6
    kvx.store_latent_rope(s.pool, s.batch, kv, theta=theta, style=style, norm=norm, norm_eps=1e-5, q=q,
                          num_q_heads=heads, q_out=q_out)
    out = torch.empty(s.T, lat + 64, dtype=BF16, device=DEV)
    kvx.load_latent(s.pool, s.batch, out)
    pos = np.concatenate([np.arange(p, p + e) for p, e in zip(P, E)])
    freqs = theta ** (-2.0 * np.arange(32) / 64)
    x = ref.f64(kv)
    c = x[:, :lat] * ref.f64(norm) / np.sqrt((x[:, :lat] ** 2).mean(-1, keepdims=True) + 1e-5)
    key = ref.rotated(x[:, lat:], pos, freqs, style)
    helpers.check_nearest_bf16(out[:, lat:].contiguous().cpu().view(torch.int16).numpy().view(np.uint16), key,
                               helpers.plane_scale(key, 64, style))
    if fp8:
        # float32 arithmetic: a value may land on the code next to it where it sits on a border
        got, e = ref.f64(out[:, :lat]), ref.scale_exps(c)
        lo = ref.quantised(c - np.abs(c) * 2.0 ** -20, e)
        hi = ref.quantised(c + np.abs(c) * 2.0 ** -20, e)
        assert ((np.minimum(lo, hi) <= got) & (got <= np.maximum(lo, hi))).all()
        assert (got != ref.quantised(c, e)).mean() < 1e-3
    else:
        helpers.check_nearest_bf16(out[:, :lat].contiguous().cpu().view(torch.int16).numpy().view(np.uint16), c, np.abs(c))
    if heads:
        want = ref.rotated(ref.f64(given[..., hd:]), pos, freqs, style)
        helpers.check_nearest_bf16(q_out[..., hd:].contiguous().cpu().view(torch.int16).numpy().view(np.uint16), want,
                                   helpers.plane_scale(want, 64, style))
        assert torch.equal(q_out[..., :hd], given[..., :hd])
        if not in_place:
            assert torch.equal(q, given)


def test_store_rope_far_positions_and_given_rates(setup):
    """Positions past 2^24, where an angle in float32 would have no digits left, with a rate table."""
    far = (1 << 27) + 3
    pages = torch.zeros(-(-(far + 2) // 16), dtype=torch.int32, device=DEV)
    s = setup([0], [16], 256, False)
    b = kvx.Batch([far], [2], [0, len(pages)], pages)
    kv = s.normal(2, 320)
    inv = np.random.default_rng(0).uniform(0, 1.5, 32)
    kvx.store_latent_rope(s.pool, b, kv, inv_freq=inv, style=1)
    out = torch.empty(2, 320, dtype=BF16, device=DEV)
    kvx.load_latent(s.pool, b, out)
    want = ref.rotated(ref.f64(kv[:, 256:]), np.array([far, far + 1]), inv, 1)
    # the angle in float64 carries 2^-53 * 2^27 * 1.5 of a radian, far below float32's rounding
    helpers.check_nearest_bf16(out[:, 256:].contiguous().cpu().view(torch.int16).numpy().view(np.uint16), want,
                               helpers.plane_scale(want, 64, 1))
    assert torch.equal(out[:, :256], kv[:, :256])


# ------------------------------------------------------------------- attention on latents

# rms: the weights' rounding and the output's, each at most 2^-8 / sqrt(3) of the value rms
RMS_ATTEND = math.sqrt(2 / 3) * 2.0 ** -8 * 1.05


def attend_and_check(s, rows, heads, scale, q=None, tag=""):
    q = s.normal(s.T, heads, s.lat + 64) if q is None else q
    out = torch.full((s.T + 1, heads, s.lat), 7.0, dtype=BF16, device=DEV)
    lse = torch.full((s.T + 1, heads), 7.0, dtype=torch.float32, device=DEV)
    kvx.latent_attention(s.pool, s.batch, q, heads, scale, out, lse)
    at = 0
    assert (out[s.T] == 7).all() and (lse[s.T] == 7).all()
    for r, (p, e) in enumerate(zip(s.P, s.E)):
        if e == 0:
            continue
        o, l, tol, ltol = ref.attend(ref.f64(q[at:at + e]), rows[r], rows[r][:, :s.lat], p, scale)
        ref.check_rows(out[at:at + e], o, tol, RMS_ATTEND, f"{tag} request {r}")
        assert (np.abs(ref.f64(lse[at:at + e]) - l) <= ltol).all(), f"{tag} request {r}: lse"
        at += e
    return out, lse


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lat,heads,P,E", [
    (512, 1, [0], [1]),                        # one key, one row
    (512, 16, [0, 62, 63, 64, 500], [1, 1, 1, 1, 1]),   # around a tile's end
    (512, 5, [100, 3, 40], [2, 0, 3]),         # rows of two 16-row blocks, a request without any
    (256, 33, [200, 17], [1, 2]),              # odd heads
    (512, 128, [129, 300], [1, 2]),            # tiles that end inside a token
    (256, 7, [0, 31], [70, 33]),               # the causal edge inside tiles
    (512, 24, [1000], [9]),
])
def test_latent_attention(setup, lat, heads, P, E, fp8):
    s = setup(P, E, lat, fp8)
    attend_and_check(s, s.fill(), heads, (128 + 64) ** -0.5)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("split", [64, 192])
def test_latent_attention_split(setup, split, fp8):
    """Forced splits, the causal edge in several parts (some of which a tile's first rows do
    not see at all)."""
    for lat, heads, P, E in ((512, 16, [700, 10, 64], [1, 1, 1]), (256, 6, [40, 300], [150, 90])):
        s = setup(P, E, lat, fp8)
        kvx.latent_pool_set_split_keys(s.pool, split)
        attend_and_check(s, s.fill(), heads, 0.07)


@pytest.mark.parametrize("heads,E", [(16, 1), (20, 1), (16, 5)])
def test_latent_attention_uneven_scores(setup, heads, E):
    """Scores from very low to very high along the keys: a late key that outweighs all before
    it by far more than float32's range of exponents, then the reverse."""
    for order in (1, -1):
        s = setup([400], [E], 512, False)
        rows = s.normal(400 + E, 576)
        rows[:, 0] = (torch.linspace(-30, 30, 400 + E, device=DEV) * order).to(BF16)
        q = s.normal(E, heads, 576, scale=0.3)
        q[..., 0] = 60.0
        attend_and_check(s, s.fill(rows=rows), heads, 0.5, q=q)


def test_latent_attention_equal_keys_and_zero_scale_rows(setup):
    """All scores equal: the mean of the values, and the log of their number."""
    s = setup([63], [1], 512, False)
    rows = s.fill()
    q = torch.zeros(1, 16, 576, dtype=BF16, device=DEV)
    out, lse = attend_and_check(s, rows, 16, 0.1, q=q)
    assert np.allclose(ref.f64(lse[0]), math.log(64), atol=1e-6)


def test_latent_attention_long(setup):
    """A cache whose slots lie past 2^31 bytes, by a page table that names its last pages."""
    n = (1 << 31) // 18432 + 40
    s = setup([500], [1], 512, False, poison=False, extra_pages=n)
    s.pages = torch.arange(s.num_pages - 32, s.num_pages, dtype=torch.int32, device=DEV)
    s.batch = kvx.Batch(s.P, s.E, s.indptr, s.pages)
    attend_and_check(s, s.fill(), 16, 0.07)


def test_latent_attention_matches_itself_on_another_stream(setup):
    s = setup([300, 800], [1, 3], 512, True)
    rows = s.fill()
    q = s.normal(s.T, 16, 576)
    a, _ = attend_and_check(s, rows, 16, 0.07, q=q)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    b = torch.empty_like(a[:s.T])
    with torch.cuda.stream(other):
        kvx.latent_attention(s.pool, s.batch, q, 16, 0.07, b)
    other.synchronize()
    assert torch.equal(a[:s.T], b)


# ------------------------------------------------------------------- per-head attention

# rms: roundings of the scores' operand, the weights, the sums or values, and the output, each
# at most 2^-8 / sqrt(3); scores of about unit size pass theirs on one to one
RMS_EXTEND = math.sqrt(4 / 3) * 2.0 ** -8 * 1.1


def extend_and_check(s, rows, heads, hd, form, tag=""):
    lat = s.lat
    q = s.normal(s.T, heads, hd + 64)
    w_uk = s.normal(heads, hd, lat, scale=lat ** -0.5)
    w_uv = s.normal(heads, hd, lat, scale=lat ** -0.5)
    scale = (hd + 64) ** -0.5
    out = torch.full((s.T + 1, heads, hd), 7.0, dtype=BF16, device=DEV)
    lse = torch.full((s.T + 1, heads), 7.0, dtype=torch.float32, device=DEV)
    kvx.latent_extend_attention(s.pool, s.batch, q, w_uk, w_uv, scale, out, lse, form=form)
    assert (out[s.T] == 7).all() and (lse[s.T] == 7).all()
    at = 0
    uk, uv = ref.f64(w_uk), ref.f64(w_uv)
    for r, (p, e) in enumerate(zip(s.P, s.E)):
        if e == 0:
            continue
        c, key = rows[r][:, :lat], rows[r][:, lat:]
        x = ref.f64(q[at:at + e])
        h = ref.HALF_BF16
        k = np.concatenate([np.einsum("hdl,jl->hjd", uk, c), np.broadcast_to(key, (heads,) + key.shape)], -1)
        v = np.einsum("hdl,jl->hjd", uv, c)
        o, l, tol, ltol = ref.attend(x, k, v, p, scale, k_err=h, v_err=h)
        # the absorbed form rounds q' = W_uk^T q and the sums in the latent space instead, where
        # the products that meet those roundings are larger: bound both
        ql = np.concatenate([np.einsum("hdl,ihd->ihl", uk, x[..., :hd]), x[..., hd:]], -1)
        o2, l2, tol2, ltol2 = ref.attend(ql, rows[r], c, p, scale, q_err=h)
        through = np.einsum("hdl,ihl->ihd", np.abs(uv), tol2 + h * (np.abs(o2) + tol2))
        ref.check_rows(out[at:at + e], o, np.maximum(tol, through), RMS_EXTEND, f"{tag} request {r}")
        assert (np.abs(ref.f64(lse[at:at + e]) - l) <= np.maximum(ltol, ltol2)).all(), f"{tag} request {r}: lse"
        at += e
    return out[:s.T]


@pytest.mark.parametrize("form", [kvx.KVX_LATENT_ABSORBED, kvx.KVX_LATENT_EXPANDED, kvx.KVX_LATENT_AUTO])
@pytest.mark.parametrize("lat,hd,heads,fp8,P,E", [
    (512, 128, 2, False, [0], [1]),
    (512, 128, 3, True, [100, 30, 0], [5, 0, 70]),
    (256, 64, 4, False, [63, 64, 65], [65, 64, 63]),
    (256, 128, 1, True, [10], [300]),          # more than one tile of tokens
    (512, 64, 5, False, [700, 3, 200], [20, 130, 1]),
])
def test_latent_extend_attention(setup, lat, hd, heads, fp8, P, E, form):
    s = setup(P, E, lat, fp8)
    extend_and_check(s, s.fill(), heads, hd, form)


def test_latent_extend_attention_split_keys(setup):
    """A few rows over many keys: both forms split their key ranges."""
    for form in (kvx.KVX_LATENT_ABSORBED, kvx.KVX_LATENT_EXPANDED):
        s = setup([6000, 50], [40, 3], 256, False)
        extend_and_check(s, s.fill(), 2, 64, form)


def test_latent_extend_many_heads_in_groups(setup):
    """Expanded keys and values of more tokens than one workspace holds for all heads at once:
    three heads go two and one.  The tokens repeat 64 cached ones, so that a softmax over those
    gives the result, and log of their number is added to lse."""
    times = (2 << 30) // (2 * 128 * 2 * 64) // 2 - 40
    L = 64 * times
    s = setup([0], [64], 256, False)
    rows = s.fill()[0]
    pages = s.pages[:4].repeat(times)
    b = kvx.Batch([L - 1], [1], [0, len(pages)], pages)
    q = s.normal(1, 3, 192)
    w_uk, w_uv = s.normal(3, 128, 256, scale=1 / 16), s.normal(3, 128, 256, scale=1 / 16)
    out = torch.empty(1, 3, 128, dtype=BF16, device=DEV)
    lse = torch.empty(1, 3, dtype=torch.float32, device=DEV)
    kvx.latent_extend_attention(s.pool, b, q, w_uk, w_uv, 0.07, out, lse, form=kvx.KVX_LATENT_EXPANDED)
    c, key, x = rows[:, :256], rows[:, 256:], ref.f64(q)
    k = np.concatenate([np.einsum("hdl,jl->hjd", ref.f64(w_uk), c), np.broadcast_to(key, (3,) + key.shape)], -1)
    v = np.einsum("hdl,jl->hjd", ref.f64(w_uv), c)
    o, l, tol, ltol = ref.attend(x, k, v, 63, 0.07, k_err=ref.HALF_BF16, v_err=ref.HALF_BF16)
    ref.check_rows(out, o, tol + np.abs(o) * L * 2.0 ** -24, RMS_EXTEND)
    assert (np.abs(ref.f64(lse) - l - math.log(times)) <= ltol + L * 2.0 ** -24).all()


# ------------------------------------------------------------------- larger plans, other orders


@pytest.mark.parametrize("fp8", [False, True])
def test_decode_of_more_requests_than_arguments_hold(setup, fp8):
    g = np.random.default_rng(3)
    P = g.integers(0, 500, 150).tolist()
    s = setup(P, [1] * 150, 256, fp8)
    attend_and_check(s, s.fill(), 12, 0.07)


def test_more_tiles_than_arguments_hold(setup):
    s = setup([100, 0, 900], [40, 70, 9], 256, True)  # 64-row tiles: 25, 44 and 6
    attend_and_check(s, s.fill(), 40, 0.07)
    kvx.latent_pool_set_split_keys(s.pool, 128)
    attend_and_check(s, s.fill(), 40, 0.07)


def test_most_heads(setup):
    s = setup([70, 5], [1, 2], 256, False)
    attend_and_check(s, s.fill(), 1024, 0.07)


def test_extend_of_more_tiles_than_arguments_hold(setup):
    s = setup([64 * i for i in range(34)], [3] * 34, 256, True)
    extend_and_check(s, s.fill(), 3, 64, kvx.KVX_LATENT_EXPANDED)
    extend_and_check(s, s.fill(), 3, 64, kvx.KVX_LATENT_ABSORBED)


def test_requests_that_share_pages(setup):
    """Two requests whose prefix is the same pages, as a prefix cache hands them out."""
    s = setup([96, 96], [5, 1], 512, True)
    first = int(s.indptr[1])
    s.pages[first:first + 6] = s.pages[:6]
    rows = s.normal(int(sum(s.P) + sum(s.E)), 576)
    rows[101:101 + 96] = rows[:96]
    kvx.store_latent(s.pool, kvx.Batch([0, 96], [101, 1], s.indptr, s.pages), torch.cat([rows[:101], rows[197:]]))
    x = ref.f64(rows)
    x[:, :512] = ref.quantised(x[:, :512])
    attend_and_check(s, [x[:101], x[101:]], 16, 0.07)
    extend_and_check(s, [x[:101], x[101:]], 2, 128, kvx.KVX_LATENT_AUTO)


@pytest.mark.parametrize("form", [kvx.KVX_LATENT_ABSORBED, kvx.KVX_LATENT_EXPANDED])
@pytest.mark.parametrize("fp8", [False, True])
def test_extend_uneven_scores(setup, fp8, form):
    """Scores that rise along the keys past what float32 exponentials of a fixed reference
    reach, and fall: the weights of all but a few keys vanish, the outputs stay those keys'."""
    for order in (1, -1):
        s = setup([300], [70], 256, fp8)
        rows = s.normal(370, 320)
        rows[:, 256] = (torch.linspace(-30, 30, 370, device=DEV) * order).to(BF16)
        x = s.fill(rows=rows)[0]
        q = s.normal(70, 2, 128, scale=0.3)
        q[..., 64] = 60.0  # times the rotated key's first value, which no form rounds
        w_uk, w_uv = s.normal(2, 64, 256, scale=1 / 16), s.normal(2, 64, 256, scale=1 / 16)
        out = torch.empty(70, 2, 64, dtype=BF16, device=DEV)
        lse = torch.empty(70, 2, dtype=torch.float32, device=DEV)
        kvx.latent_extend_attention(s.pool, s.batch, q, w_uk, w_uv, 0.5, out, lse, form=form)
        c, key, h = x[:, :256], x[:, 256:], ref.HALF_BF16
        uk, uv, qq = ref.f64(w_uk), ref.f64(w_uv), ref.f64(q)
        v = np.einsum("hdl,jl->hjd", uv, c)
        # only the products with the expanded part (or with q') meet a rounding: bound those apart
        k = np.concatenate([np.einsum("hdl,jl->hjd", uk, c), np.broadcast_to(key, (2,) + key.shape)], -1)
        o, l, tol, ltol = ref.attend(qq, k, v, 300, 0.5, v_err=h)
        ql = np.einsum("hdl,ihd->ihl", uk, qq[..., :64])
        size = np.maximum(np.einsum("ihd,hjd->ihj", np.abs(qq[..., :64]), np.abs(k[..., :64])),
                          np.einsum("ihl,jl->ihj", np.abs(ql), np.abs(c))).max(-1) * 0.5 * h
        a = np.einsum("ihj,hjd->ihd", np.exp(np.where(np.arange(370)[None, None] <= 300 + np.arange(70)[:, None, None],
                                                      np.einsum("ihd,hjd->ihj", qq, k) * 0.5, -np.inf) - l[..., None]),
                      np.abs(v))
        tol = tol + a * np.expm1(2 * size)[..., None]
        if form == kvx.KVX_LATENT_ABSORBED:  # the sums in the latent space are rounded instead of the values
            sums = np.einsum("ihj,jl->ihl", np.exp(np.where(np.arange(370)[None, None] <= 300 + np.arange(70)[:, None, None],
                                                            np.einsum("ihd,hjd->ihj", qq, k) * 0.5, -np.inf) - l[..., None]),
                             np.abs(c))
            tol = tol + np.einsum("hdl,ihl->ihd", np.abs(uv), sums * (2 * h + np.expm1(2 * size)[..., None]))
        got = ref.f64(out)
        assert np.isfinite(got).all() and (np.abs(got - o) <= tol + h * (np.abs(o) + tol)).all()
        assert (np.abs(ref.f64(lse) - l) <= ltol + size).all()


def test_uneven_scores_of_8_bit_latents(setup):
    for order, heads, E in ((1, 16, 1), (-1, 16, 1), (1, 33, 2), (1, 30, 1)):
        s = setup([700], [E], 512, True)
        rows = s.normal(700 + E, 576)
        rows[:, 512] = (torch.linspace(-30, 30, 700 + E, device=DEV) * order).to(BF16)
        q = s.normal(E, heads, 576, scale=0.3)
        q[..., 512] = 60.0
        attend_and_check(s, s.fill(rows=rows), heads, 0.5, q=q)


def test_auto_takes_both_forms_in_one_call(setup):
    """Decoding requests on both sides of a long prompt: the prompt goes expanded, the others
    absorbed, and every row lands where it belongs."""
    lat, hd, heads, n = 256, 64, 32, 2500
    P, E = [3000] * 12 + [0] + [3000] * 12, [1] * 12 + [n] + [2] * 12
    s = setup(P, E, lat, False)
    rows = s.fill()
    q = s.normal(s.T, heads, hd + 64)
    w_uk, w_uv = s.normal(heads, hd, lat, scale=1 / 16), s.normal(heads, hd, lat, scale=1 / 16)
    out = torch.full((s.T + 1, heads, hd), 7.0, dtype=BF16, device=DEV)
    lse = torch.full((s.T + 1, heads), 7.0, dtype=torch.float32, device=DEV)
    kvx.latent_extend_attention(s.pool, s.batch, q, w_uk, w_uv, 0.09, out, lse)
    assert (out[s.T] == 7).all() and (lse[s.T] == 7).all()
    uk, uv, at = ref.f64(w_uk), ref.f64(w_uv), 0
    for r, (p, e) in enumerate(zip(P, E)):
        take = 3  # of the prompt its last rows
        first = at + max(e - take, 0)
        x, c = ref.f64(q[first:at + e]), rows[r][:, :lat]
        k = np.concatenate([np.einsum("hdl,jl->hjd", uk, c), np.broadcast_to(rows[r][:, lat:], (heads,) + rows[r][:, lat:].shape)], -1)
        o, l, _, _ = ref.attend(x, k, np.einsum("hdl,jl->hjd", uv, c), p + max(e - take, 0), 0.09)
        got = ref.f64(out[first:at + e])
        assert np.linalg.norm(got - o) <= RMS_EXTEND * np.linalg.norm(o), r
        # a score carries one rounding of 64 products' factor: of rms 2^-8 / sqrt(3) of its size
        assert np.abs(ref.f64(lse[first:at + e]) - l).max() < 2.0 ** -8
        at += e


def test_forms_agree_and_calls_repeat(setup):
    """The same call twice gives the same bits, with or without lse; the two forms differ by
    their roundings only."""
    s = setup([500, 0, 2000], [3, 90, 1], 512, True)
    s.fill()
    q = s.normal(s.T, 16, 192)
    w_uk, w_uv = s.normal(16, 128, 512, scale=512 ** -0.5), s.normal(16, 128, 512, scale=512 ** -0.5)

    def call(form, with_lse=True):
        out = torch.empty(s.T, 16, 128, dtype=BF16, device=DEV)
        lse = torch.empty(s.T, 16, dtype=torch.float32, device=DEV) if with_lse else None
        kvx.latent_extend_attention(s.pool, s.batch, q, w_uk, w_uv, 0.07, out, lse, form=form)
        return out, lse

    got = {}
    for form in (kvx.KVX_LATENT_ABSORBED, kvx.KVX_LATENT_EXPANDED, kvx.KVX_LATENT_AUTO):
        got[form] = call(form)
        again = call(form)
        assert torch.equal(got[form][0], again[0]) and torch.equal(got[form][1], again[1])
        assert torch.equal(got[form][0], call(form, False)[0])
    a, b = (got[f][0].float() for f in (kvx.KVX_LATENT_ABSORBED, kvx.KVX_LATENT_EXPANDED))
    assert (a - b).norm() <= 2 * RMS_EXTEND * b.norm()


def test_two_pools_on_two_streams(setup):
    pools = [setup([400 + 100 * i, 30], [1, 20], 256, bool(i), seed=i) for i in range(2)]
    args = []
    for s in pools:
        s.fill()
        args.append((s.normal(s.T, 24, 320), torch.empty(s.T, 24, 256, dtype=BF16, device=DEV)))
        kvx.latent_attention(s.pool, s.batch, args[-1][0], 24, 0.07, args[-1][1])
    torch.cuda.synchronize()
    want = [o.clone() for _, o in args]
    streams = [torch.cuda.Stream() for _ in pools]
    for _ in range(3):
        for s, (q, o), st in zip(pools, args, streams):
            with torch.cuda.stream(st):
                o.zero_()
                kvx.latent_attention(s.pool, s.batch, q, 24, 0.07, o)
        torch.cuda.synchronize()
        for (_, o), w in zip(args, want):
            assert torch.equal(o, w)


def test_empty_batches(setup):
    s = setup([20, 0], [0, 0], 256, False, poison=False)
    nothing = kvx.Batch([], [], [0], torch.empty(0, dtype=torch.int32, device=DEV))
    for b in (s.batch, nothing):
        x = torch.empty(0, 320, dtype=BF16, device=DEV)
        kvx.store_latent(s.pool, b, x)
        kvx.load_latent(s.pool, b, x)
        kvx.latent_attention(s.pool, b, torch.empty(0, 4, 320, dtype=BF16, device=DEV), 4, 0.1,
                             torch.empty(0, 4, 256, dtype=BF16, device=DEV))


# ------------------------------------------------------------------- refusals


def test_capturing_stream_is_refused(setup):
    s = setup([40], [2], 256, False)
    s.fill()
    q, o = s.normal(2, 4, 320), torch.empty(2, 4, 256, dtype=BF16, device=DEV)
    row, x = s.normal(2, 320), torch.zeros(4, device=DEV)
    w = s.normal(4, 64, 256)
    qs, os_ = s.normal(2, 4, 128), torch.empty(2, 4, 64, dtype=BF16, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x += 1
        for call in (lambda: kvx.store_latent(s.pool, s.batch, row), lambda: kvx.load_latent(s.pool, s.batch, row),
                     lambda: kvx.store_latent_rope(s.pool, s.batch, row),
                     lambda: kvx.latent_attention(s.pool, s.batch, q, 4, 0.1, o),
                     lambda: kvx.latent_extend_attention(s.pool, s.batch, qs, w, w, 0.1, os_)):
            with pytest.raises(kvx.KvxError) as e:
                call()
            assert e.value.status == kvx.KVX_EUNSUPPORTED
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert (x == 2).all()


def test_validation_names_bad_pages(setup, monkeypatch):
    s = setup([40], [2], 256, False)
    monkeypatch.setenv("KVX_VALIDATE", "1")
    row = s.normal(2, 320)
    kvx.store_latent(s.pool, s.batch, row)
    for bad in (s.num_pages, -1):
        s.pages[1] = bad
        b = kvx.Batch(s.P, s.E, s.indptr, s.pages)
        w, q = s.normal(4, 64, 256), s.normal(2, 4, 320)
        for call in (lambda: kvx.store_latent(s.pool, b, row), lambda: kvx.load_latent(s.pool, b, row),
                     lambda: kvx.store_latent_rope(s.pool, b, row),
                     lambda: kvx.latent_attention(s.pool, b, q, 4, 0.1, q.clone()),
                     lambda: kvx.latent_extend_attention(s.pool, b, q, w, w, 0.1, q.clone())):
            with pytest.raises(kvx.KvxError) as e:
                call()
            assert e.value.status == kvx.KVX_ERANGE


def test_pool_that_does_not_fit():
    with pytest.raises(kvx.KvxError) as e:
        kvx.latent_pool_create((1 << 31) - 1, 16, 512, 64, kvx.KVX_LATENT_BF16)  # 39 TB
    assert e.value.status == kvx.KVX_ENOMEM
    assert (torch.ones(8, device=DEV) + 1).sum().item() == 16  # the failure is not found by other calls

# ------------------------------------------------------------------- together

def test_turns_of_agents(setup):
    """A prompt, a short turn and drafted tokens of several agents over one pool: each step
    stores and attends as a layer does, in both forms, against attention over whole sequences."""
    lat, hd, heads = 256, 64, 4
    lens = [(90, 12, 3, 1), (33, 40, 1, 1), (7, 1, 2, 5)]
    total = [sum(x) for x in lens]
    s = setup([0] * 3, total, lat, False)
    kv = s.normal(sum(total), lat + 64)
    q = s.normal(sum(total), heads, hd + 64)
    norm = 1.0 + s.normal(lat, scale=0.2)
    w_uk, w_uv = s.normal(heads, hd, lat, scale=1 / 16), s.normal(heads, hd, lat, scale=1 / 16)
    base = np.cumsum([0] + total)
    scale = (hd + 64) ** -0.5
    got = torch.empty(sum(total), heads, hd, dtype=BF16, device=DEV)
    turned = torch.empty_like(q)
    done = [0, 0, 0]
    for step in range(4):
        E = [x[step] for x in lens]
        at = torch.cat([torch.arange(base[i] + done[i], base[i] + done[i] + E[i]) for i in range(3)]).to(DEV)
        b = kvx.Batch(done, E, s.indptr, s.pages)
        qs = torch.empty(len(at), heads, hd + 64, dtype=BF16, device=DEV)
        kvx.store_latent_rope(s.pool, b, kv[at], norm=norm, q=q[at], num_q_heads=heads, q_out=qs)
        o = torch.empty(len(at), heads, hd, dtype=BF16, device=DEV)
        kvx.latent_extend_attention(s.pool, b, qs, w_uk, w_uv, scale, o)
        got[at], turned[at] = o, qs
        done = [d + e for d, e in zip(done, E)]
    rows = torch.empty(sum(total), lat + 64, dtype=BF16, device=DEV)
    kvx.load_latent(s.pool, kvx.Batch([0] * 3, total, s.indptr, s.pages), rows)
    for i in range(3):
        r = ref.f64(rows[base[i]:base[i + 1]])
        k = np.concatenate([np.einsum("hdl,jl->hjd", ref.f64(w_uk), r[:, :lat]),
                            np.broadcast_to(r[:, lat:], (heads, total[i], 64))], -1)
        v = np.einsum("hdl,jl->hjd", ref.f64(w_uv), r[:, :lat])
        o, _, tol, _ = ref.attend(ref.f64(turned[base[i]:base[i + 1]]), k, v, 0, scale, k_err=ref.HALF_BF16,
                                  v_err=ref.HALF_BF16)
        g = ref.f64(got[base[i]:base[i + 1]])
        assert np.linalg.norm(g - o) <= RMS_EXTEND * np.linalg.norm(o)


def test_agents_through_the_prefix_cache():
    """Agents whose histories the round-robin prefix cache keeps in a latent pool that is too small
    for all: prefixes that stayed are attended where they lie, what was evicted is stored again."""
    lat, hd, heads, num_pages = 256, 64, 3, 60
    pool = kvx.latent_pool_create(num_pages, 16, lat, 64, kvx.KVX_LATENT_FP8)
    cache = kvx.kvx_cache_create(num_pages, 16, 64, kvx.KVX_EVICT_RR)
    g = torch.Generator(DEV).manual_seed(11)
    rng = np.random.default_rng(11)
    kv = [torch.randn(600, lat + 64, device=DEV, generator=g, dtype=BF16) for _ in range(4)]
    w_uk, w_uv = (torch.randn(heads, hd, lat, device=DEV, generator=g, dtype=BF16) / 16 for _ in range(2))
    uk, uv, scale = ref.f64(w_uk), ref.f64(w_uv), (hd + 64) ** -0.5
    lens, reused, missed = [0] * 4, 0, 0
    try:
        for turn in range(5):
            for agent in range(4):
                before = lens[agent]
                lens[agent] += int(rng.integers(40, 110))
                prefix, table = kvx.kvx_cache_begin_turn(cache, agent, lens[agent])
                reused, missed = reused + prefix, missed + before - min(prefix, before)
                e = lens[agent] - prefix
                b = kvx.Batch([prefix], [e], [0, len(table)], torch.from_numpy(table).to(DEV))
                q = torch.randn(e, heads, hd + 64, device=DEV, generator=g, dtype=BF16)
                out = torch.empty(e, heads, hd, dtype=BF16, device=DEV)
                turned = torch.empty_like(q)
                kvx.store_latent_rope(pool, b, kv[agent][prefix:lens[agent]], q=q, num_q_heads=heads, q_out=turned)
                kvx.latent_extend_attention(pool, b, turned, w_uk, w_uv, scale, out)
                kvx.kvx_cache_end_turn(cache, agent)
                # the whole history from its own rows, not from the pool
                x, pos = ref.f64(kv[agent][:lens[agent]]), np.arange(lens[agent])
                freqs = 10000.0 ** (-2.0 * np.arange(32) / 64)
                c = ref.quantised(x[:, :lat])
                r = ref.rotated(x[:, lat:], pos, freqs, 0)
                k = np.concatenate([np.einsum("hdl,jl->hjd", uk, c), np.broadcast_to(r, (heads,) + r.shape)], -1)
                qr = ref.f64(q)
                qr[..., hd:] = ref.rotated(qr[..., hd:], pos[prefix:], freqs, 0)
                o, _, _, _ = ref.attend(qr, k, np.einsum("hdl,jl->hjd", uv, c), prefix, scale)
                # RMS_EXTEND's four roundings and those of the rotated halves of keys and queries
                assert np.linalg.norm(ref.f64(out) - o) <= RMS_EXTEND * math.sqrt(6 / 4) * np.linalg.norm(o), (turn, agent)
        assert reused > 0 and missed > 0
    finally:
        torch.cuda.synchronize()
        kvx.kvx_cache_destroy(cache)
        kvx.latent_pool_destroy(pool)


# ------------------------------------------------------------------- scores past float32


def overflowing(s, heads, dim, low, scale=0.3):
    """Cached rows and queries whose first 64 scores lie below float32's range (-1.2e39, from the
    first rotated dim), the others `low` (from the second) plus what the rest of the dims give."""
    rows = s.normal(sum(s.P) + sum(s.E), s.lat + 64)
    rows[:64, s.lat], rows[64:, s.lat] = -4.0, 0.0
    rows[:, s.lat + 1] = -low / 16
    q = s.normal(s.T, heads, dim, scale=scale)
    q[..., -64], q[..., -63] = 3e38, 16.0
    return rows, q


@pytest.mark.parametrize("low", [0, 4096])
@pytest.mark.parametrize("split", [0, 64, 192, 1024])
@pytest.mark.parametrize("heads,E,fp8", [(16, 1, False), (20, 1, True), (16, 5, False), (33, 3, True)])
def test_latent_attention_after_scores_below_float32(setup, heads, E, fp8, split, low):
    """Keys whose scores overflow to -inf have no weight; the keys after them count in full, also
    where they lie so low that exponentials against a reference of zero would vanish."""
    s = setup([400], [E], 256, fp8)
    kvx.latent_pool_set_split_keys(s.pool, split)
    rows, q = overflowing(s, heads, 320, low)
    x = s.fill(rows=rows)[0]
    out = torch.empty(E, heads, 256, dtype=BF16, device=DEV)
    lse = torch.empty(E, heads, dtype=torch.float32, device=DEV)
    kvx.latent_attention(s.pool, s.batch, q, heads, 0.07, out, lse)
    o, l, tol, ltol = ref.attend(ref.f64(q), x[64:], x[64:, :256], 400 - 64, 0.07)
    # scores of 4096 * 0.07 carry float32 steps of 2^-15, which the rms of the roundings does not see
    ref.check_rows(out, o, tol, RMS_ATTEND)
    assert (np.abs(ref.f64(lse) - l) <= ltol).all()


@pytest.mark.parametrize("low", [0, 4096])
@pytest.mark.parametrize("form", [kvx.KVX_LATENT_ABSORBED, kvx.KVX_LATENT_EXPANDED])
@pytest.mark.parametrize("hd,P,E", [(64, 400, 70), (128, 6000, 40)])  # the second splits its keys
def test_extend_after_scores_below_float32(setup, hd, P, E, form, low):
    s = setup([P], [E], 256, False)
    rows, q = overflowing(s, 2, hd + 64, low)
    x = s.fill(rows=rows)[0][64:]
    w_uk, w_uv = s.normal(2, hd, 256, scale=1 / 16), s.normal(2, hd, 256, scale=1 / 16)
    out = torch.empty(E, 2, hd, dtype=BF16, device=DEV)
    lse = torch.empty(E, 2, dtype=torch.float32, device=DEV)
    kvx.latent_extend_attention(s.pool, s.batch, q, w_uk, w_uv, 0.07, out, lse, form=form)
    uk, uv, qq, c = ref.f64(w_uk), ref.f64(w_uv), ref.f64(q), x[:, :256]
    k = np.concatenate([np.einsum("hdl,jl->hjd", uk, c), np.broadcast_to(x[:, 256:], (2, len(x), 64))], -1)
    o, l, _, _ = ref.attend(qq, k, np.einsum("hdl,jl->hjd", uv, c), P - 64, 0.07)
    got = ref.f64(out)
    assert np.isfinite(got).all() and np.linalg.norm(got - o) <= RMS_EXTEND * np.linalg.norm(o)
    # half a bf16 step of every term of the products that meet a rounding (the rotated dims meet none)
    ql = np.einsum("hdl,ihd->ihl", uk, qq[..., :hd])
    size = np.maximum(np.einsum("ihd,hjd->ihj", np.abs(qq[..., :hd]), np.abs(k[..., :hd])),
                      np.einsum("ihl,jl->ihj", np.abs(ql), np.abs(c))).max(-1) * 0.07 * ref.HALF_BF16
    rest = (np.abs(l) + low * 0.07 + 30.0) * (320 + P) * ref.F32  # float32 sums of up to 320 terms and P weights
    assert (np.abs(ref.f64(lse) - l) <= size + rest).all()


@pytest.mark.parametrize("split", [0, 64])
@pytest.mark.parametrize("key", [5, 170])
def test_scores_above_float32_give_nan(setup, split, key):
    """A scaled score past float32's largest value: NaN in its row, as inf - inf is, and in no other."""
    s = setup([300], [1], 256, False)
    kvx.latent_pool_set_split_keys(s.pool, split)
    rows = s.normal(301, 320)
    rows[:, 256] = 0.0
    rows[key, 256] = 1e10
    x = s.fill(rows=rows)[0]
    w_uk, w_uv = s.normal(4, 64, 256, scale=1 / 16), s.normal(4, 64, 256, scale=1 / 16)

    def check(dim, width, v, call, rms):
        q = torch.zeros(1, 4, dim, dtype=BF16, device=DEV)
        q[0, 2, -64] = 1e10
        out = torch.zeros(1, 4, width, dtype=BF16, device=DEV)
        lse = torch.zeros(1, 4, dtype=torch.float32, device=DEV)
        call(q, out, lse)
        got, l = ref.f64(out)[0], ref.f64(lse)[0]
        assert np.isnan(got[2]).all() and np.isnan(l[2])
        others = [0, 1, 3]
        want = (v if v.ndim == 3 else np.broadcast_to(v, (4,) + v.shape)).mean(1)
        assert np.linalg.norm(got[others] - want[others]) <= rms * np.linalg.norm(want[others])
        assert np.abs(l[others] - math.log(301)).max() < 1e-5

    check(320, 256, x[:, :256], lambda q, o, l: kvx.latent_attention(s.pool, s.batch, q, 4, 1e20, o, l), RMS_ATTEND)
    v = np.einsum("hdl,jl->hjd", ref.f64(w_uv), x[:, :256])
    for form in (kvx.KVX_LATENT_ABSORBED, kvx.KVX_LATENT_EXPANDED):
        check(128, 64, v, lambda q, o, l: kvx.latent_extend_attention(s.pool, s.batch, q, w_uk, w_uv, 1e20, o, l, form=form),
              RMS_EXTEND)


@pytest.mark.parametrize("split", [0, 64])
def test_rows_without_a_score_and_nan_queries(setup, split):
    """A head whose scores are all -inf gives zeros and an lse of -inf, one with a NaN in its query
    NaN; the heads beside them in the same unit are what they are without."""
    s = setup([300], [2], 256, True)
    kvx.latent_pool_set_split_keys(s.pool, split)
    rows = s.normal(302, 320)
    rows[:, 256] = -4.0
    s.fill(rows=rows)
    w_uk, w_uv = s.normal(5, 64, 256, scale=1 / 16), s.normal(5, 64, 256, scale=1 / 16)

    def check(dim, width, call):
        q = s.normal(2, 5, dim)
        got = []
        for spoil in (False, True):
            if spoil:
                q[:, 1, -64], q[:, 3, 7] = 3e38, math.nan
            out = torch.full((2, 5, width), 7.0, dtype=BF16, device=DEV)
            lse = torch.full((2, 5), 7.0, dtype=torch.float32, device=DEV)
            call(q, out, lse)
            got.append((ref.f64(out), ref.f64(lse)))
        (o, l), (po, pl) = got
        assert (po[:, 1] == 0).all() and (pl[:, 1] == -math.inf).all()
        assert np.isnan(po[:, 3]).all() and np.isnan(pl[:, 3]).all()
        # a unit that is run again has another reference point: the roundings of the weights differ
        for h in (0, 2, 4):
            assert np.linalg.norm(po[:, h] - o[:, h]) <= 2 * RMS_EXTEND * np.linalg.norm(o[:, h])
            # two float32 sums of 302 weights
            assert np.abs(pl[:, h] - l[:, h]).max() <= 2 * (302 + 16) * ref.F32

    check(320, 256, lambda q, o, l: kvx.latent_attention(s.pool, s.batch, q, 5, 0.07, o, l))
    for form in (kvx.KVX_LATENT_ABSORBED, kvx.KVX_LATENT_EXPANDED):
        check(128, 64, lambda q, o, l: kvx.latent_extend_attention(s.pool, s.batch, q, w_uk, w_uv, 0.09, o, l, form=form))


# ------------------------------------------------------------------- many heads of one expansion


def heads_a_workgroup(units, heads):
    """Heads that a workgroup of the expansion takes one after the other: the number that ends
    first on 256 CUs at a head's time each and half a head's time for the tokens, the largest such."""
    return min(range(heads, 0, -1), key=lambda per: -(-units * -(-heads // per) // 256) * (per + 0.5))


@pytest.mark.parametrize("lat,hd,heads,fp8", [
    (512, 128, 17, False), (512, 128, 17, True), (512, 64, 23, True), (512, 64, 17, False), (256, 128, 17, True),
    (256, 64, 29, False)])
def test_expansion_of_several_heads_a_workgroup(setup, lat, hd, heads, fp8):
    """Each workgroup forms the keys and values of three heads or more, the last of them of fewer:
    operands, stores and waits run on from one head to the next."""
    g = np.random.default_rng(lat + hd + heads)
    E = g.integers(1, 4, 36).tolist()
    P = [int(x) - e for x, e in zip(g.integers(4, 120, 36), E)]
    P[3], P[4] = 256 - E[3], 256  # a whole unit, and one token or a few past it
    units = sum(-(-(p + e) // 256) for p, e in zip(P, E))
    per = heads_a_workgroup(units, heads)
    assert per >= 3 and heads % per != 0
    s = setup(P, E, lat, fp8)
    rows = s.fill()
    q = s.normal(s.T, heads, hd + 64)
    w_uk, w_uv = (s.normal(heads, hd, lat, scale=lat ** -0.5) for _ in range(2))
    out = torch.full((s.T + 1, heads, hd), 7.0, dtype=BF16, device=DEV)
    lse = torch.full((s.T + 1, heads), 7.0, dtype=torch.float32, device=DEV)
    scale = (hd + 64) ** -0.5
    kvx.latent_extend_attention(s.pool, s.batch, q, w_uk, w_uv, scale, out, lse, form=kvx.KVX_LATENT_EXPANDED)
    assert (out[s.T] == 7).all() and (lse[s.T] == 7).all()
    qq, uk, uv, at = ref.f64(q), ref.f64(w_uk).reshape(-1, lat), ref.f64(w_uv).reshape(-1, lat), 0
    for r, (p, e) in enumerate(zip(P, E)):
        c, key = rows[r][:, :lat], rows[r][:, lat:]
        k = (c @ uk.T).reshape(-1, heads, hd).transpose(1, 0, 2)
        k = np.concatenate([k, np.broadcast_to(key, (heads,) + key.shape)], -1)
        v = (c @ uv.T).reshape(-1, heads, hd).transpose(1, 0, 2)
        o, l, tol, ltol = ref.attend(qq[at:at + e], k, v, p, scale, k_err=ref.HALF_BF16, v_err=ref.HALF_BF16)
        ref.check_rows(out[at:at + e], o, tol, RMS_EXTEND, f"request {r}")
        assert (np.abs(ref.f64(lse[at:at + e]) - l) <= ltol).all(), f"request {r}: lse"
        at += e


@pytest.mark.parametrize("lat,hd,fp8", [(512, 128, True), (256, 64, False)])
def test_rows_throughout_a_long_suffix(setup, lat, hd, fp8):
    """A suffix of several tiles of tokens, split keys and several heads a workgroup: the first and
    last rows, those around every tile's border and some in between."""
    P, n, heads = 1500, 2300, 35
    s = setup([P], [n], lat, fp8)
    rows = s.fill()[0]
    per = heads_a_workgroup(-(-(P + n) // 256), heads)
    assert per >= 2
    q = s.normal(n, heads, hd + 64)
    w_uk, w_uv = (s.normal(heads, hd, lat, scale=lat ** -0.5) for _ in range(2))
    out = torch.empty(n, heads, hd, dtype=BF16, device=DEV)
    lse = torch.empty(n, heads, dtype=torch.float32, device=DEV)
    scale = (hd + 64) ** -0.5
    kvx.latent_extend_attention(s.pool, s.batch, q, w_uk, w_uv, scale, out, lse, form=kvx.KVX_LATENT_EXPANDED)
    picks = sorted({0, 1, n - 1} | {t + i for t in range(256, n, 256) for i in (-1, 0)} |
                   set(np.random.default_rng(1).integers(0, n, 12).tolist()))
    c, key = rows[:, :lat], rows[:, lat:]
    k = (c @ ref.f64(w_uk).reshape(-1, lat).T).reshape(-1, heads, hd).transpose(1, 0, 2)
    k = np.concatenate([k, np.broadcast_to(key, (heads,) + key.shape)], -1)
    v = (c @ ref.f64(w_uv).reshape(-1, lat).T).reshape(-1, heads, hd).transpose(1, 0, 2)
    for i in picks:
        o, l, tol, ltol = ref.attend(ref.f64(q[i:i + 1]), k[:, :P + i + 1], v[:, :P + i + 1], P + i, scale,
                                     k_err=ref.HALF_BF16, v_err=ref.HALF_BF16)
        ref.check_rows(out[i:i + 1], o, tol, RMS_EXTEND, f"row {i}")
        assert (np.abs(ref.f64(lse[i:i + 1]) - l) <= ltol).all(), f"row {i}: lse"
