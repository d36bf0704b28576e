"""Cross attention on the GPU against a float64 reference (tests/page_ref.py), on every pool type:
queries of one length over states of another, single queries and many, requests without
states, odd sizes and pages that end inside a tile."""

import math

import numpy as np
import pytest
import torch

import page_ref as ref
from paper_2609_32278_amd import kvx
from test_gpu_page_pool import BF16, DEV, setup  # noqa: F401

pytestmark = pytest.mark.gpu
POOLS = [kvx.KVX_KV_BF16, kvx.KVX_KV_FP8_E4M3, kvx.KVX_KV_FP8_PAGE]


def run(s, held, group, scale, err=0.0, lse=True, tag=""):
    hq = s.hkv * group
    q = s.normal(s.T, hq, s.d)
    out = torch.full((s.T + 1, hq, s.d), 7.0, dtype=BF16, device=DEV)
    ls = torch.full((s.T + 1, hq), 7.0, device=DEV)
    print(f"[cross] {tag} L={s.P} E={s.E} hkv={s.hkv} group={group} d={s.d} pool={s.dtype}", flush=True)
    kvx.cross_attention(s.pool, s.batch, q, hq, scale, out[:s.T], ls[:s.T] if lse else None)
    torch.cuda.synchronize()
    assert (out[s.T:] == 7).all() and (ls[s.T:] == 7).all()
    at = 0
    for r, e in enumerate(s.E):
        o, l, to, tl = ref.attend(ref.f64(q[at:at + e]), *held[r], scale, q_err=err)
        if s.P[r] == 0:
            assert (out[at:at + e].view(torch.int16) == 0).all() and (not lse or (ls[at:at + e] == -math.inf).all())
        else:
            ref.check(ref.f64(out[at:at + e]), o, to, f"request {r}")
            if lse:
                ref.check(ref.f64(ls[at:at + e]), l, tl, f"lse of request {r}")
        at += e
    return q, out[:s.T], ls[:s.T]


CASES = [
    # L, E, hkv, group
    ([1], [1], 1, 1),
    ([16, 15, 17, 1], [1, 2, 3, 16], 2, 1),
    ([64, 63, 65, 0, 129], [16, 17, 33, 5, 0], 1, 1),
    ([300, 40], [2, 3], 2, 5),
    ([200, 0, 77], [4, 100, 9], 3, 4),
    ([1000, 31], [300, 64], 2, 4),
    ([90, 700], [1, 2], 2, 16),
    ([50, 0, 333], [1, 7, 40], 1, 20),           # more heads on a KV head than the decode code takes
    ([512], [257], 8, 1),
]


@pytest.mark.parametrize("dtype", POOLS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("L,E,hkv,group", CASES)
def test_cross(setup, L, E, hkv, group, d, dtype):  # noqa: F811
    s = setup(L, E, hkv, d, dtype, cross=True)
    held = s.fill(lens=L)
    run(s, held, group, 1 / math.sqrt(d))
    run(s, held, group, 1 / math.sqrt(d), lse=False)
    kvx.kv_pool_set_split_keys(s.pool, 64)
    run(s, held, group, 1 / math.sqrt(d), tag="split")
    kvx.kv_pool_set_split_keys(s.pool, 0)
    kvx.kv_pool_set_scaled_q(s.pool, True)
    run(s, held, group, 1 / math.sqrt(d), ref.HALF_BF16, tag="scaled Q")


@pytest.mark.parametrize("dtype", POOLS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,tokens", [(1, 64), (1, 65), (1, 96), (1, 128), (1, 129), (3, 33), (8, 16), (8, 17), (32, 4), (33, 3)])
def test_as_entries_and_as_tiles(setup, dtype, d, group, tokens):  # noqa: F811
    """Around the numbers of rows where a batch changes from entries of 32 rows to tiles."""
    s = setup([333, 70], [tokens, 1], 2, d, dtype, cross=True)
    run(s, s.fill(lens=s.P), group, 0.1)


@pytest.mark.parametrize("dtype", POOLS)
@pytest.mark.parametrize("e", [1, 3, 200])
@pytest.mark.parametrize("split", [0, 64])
def test_a_nan_query_stays_in_its_row(setup, dtype, e, split):  # noqa: F811
    s = setup([300, 90], [e, e], 2, 64, dtype, cross=True)
    s.fill(lens=s.P)
    kvx.kv_pool_set_split_keys(s.pool, split)
    q = s.normal(s.T, 8, 64)
    bad = q.clone()
    bad[e - 1, 3, 5] = float("nan")
    out, good = torch.empty_like(q), torch.empty_like(q)
    kvx.cross_attention(s.pool, s.batch, bad, 8, 0.125, out)
    kvx.cross_attention(s.pool, s.batch, q, 8, 0.125, good)
    rest = torch.ones(s.T, 8, dtype=torch.bool, device=DEV)
    rest[e - 1, 3] = False
    assert torch.isnan(out[e - 1, 3]).all() and torch.isfinite(good).all()
    assert torch.equal(out[rest], good[rest])


@pytest.mark.parametrize("dtype", POOLS)
@pytest.mark.parametrize("e", [1, 3, 20])
def test_many_requests(setup, dtype, e):  # noqa: F811
    """More requests than the kernel arguments hold, some without states, some without queries."""
    L = [0 if i % 7 == 0 else (i * 53) % 400 + 1 for i in range(260)]
    E = [0 if i % 11 == 0 else e for i in range(260)]
    s = setup(L, E, 3, 64, dtype, cross=True)
    run(s, s.fill(lens=L), 2, 0.125)


@pytest.mark.parametrize("dtype", POOLS)
def test_long_states(setup, dtype):  # noqa: F811
    """Ranges that are split by themselves: few queries over long states, and prompts beside steps."""
    L, E = [9001, 20000, 4097], [1, 2, 70]
    s = setup(L, E, 2, 128, dtype, cross=True)
    run(s, s.fill(lens=L), 4, 0.08)


@pytest.mark.parametrize("dtype", POOLS)
@pytest.mark.parametrize("e", [2, 200])
def test_scores_far_above_the_first_tile(setup, dtype, e):  # noqa: F811
    L = [500]
    s = setup(L, [e], 1, 128, dtype, cross=True)
    k, v = s.normal(500, 1, 128), s.normal(500, 1, 128)
    if dtype != kvx.KVX_KV_FP8_E4M3:  # static scales hold no such values
        k[200] *= 40.0
        k[499] *= 90.0
    run(s, s.fill(lens=L, seed_rows=(k, v)), 4, 1.0)


@pytest.mark.parametrize("dtype", POOLS)
def test_states_that_requests_share(setup, dtype):  # noqa: F811
    """Requests that attend to one encoding: the same pages listed for each."""
    s = setup([130, 130, 130], [1, 1, 40], 2, 64, dtype, cross=True)
    pages = np.concatenate([s.pages_of(0)] * 3).astype(np.int32)
    s.host_pages, s.pages = pages, torch.from_numpy(pages).to(DEV)
    s.batch = kvx.Batch(s.P, s.E, s.indptr, s.pages)
    k, v = s.normal(130, 2, 64), s.normal(130, 2, 64)
    held = s.fill(lens=[130, 0, 0], seed_rows=(k, v))
    run(s, [held[0]] * 3, 3, 0.125)


def test_one_query_is_the_decode_step(setup):  # noqa: F811
    """A single query over L tokens is extend_attention's over a prefix of L - 1 and itself."""
    for dtype in POOLS:
        s = setup([40, 700, 129], [1, 1, 1], 2, 128, dtype, cross=True)
        held = s.fill(lens=s.P)
        q = s.normal(3, 8, 128)
        a, b = torch.empty_like(q), torch.empty_like(q)
        kvx.cross_attention(s.pool, s.batch, q, 8, 0.1, a)
        kvx.extend_attention(s.pool, kvx.Batch([39, 699, 128], [1, 1, 1], s.indptr, s.pages), q, 8, 0.1, b)
        for r in range(3):
            o, _, to, _ = ref.attend(ref.f64(q[r:r + 1]), *held[r], 0.1)
            for got in (a, b):
                ref.check(ref.f64(got[r:r + 1]), o, to, f"request {r}")
        if dtype == kvx.KVX_KV_FP8_PAGE:  # the same code takes both
            assert torch.equal(a, b)


def test_no_queries_and_no_states(setup):  # noqa: F811
    s = setup([0, 0], [3, 1200], 2, 64, kvx.KVX_KV_BF16, cross=True)
    run(s, s.fill(lens=[0, 0]), 24, 0.125)
    none = kvx.Batch([5, 0], [0, 0], [0, 1, 1], s.pages)
    kvx.cross_attention(s.pool, none, s.normal(1, 4, 64), 4, 0.1, s.normal(1, 4, 64))
    kvx.cross_attention(s.pool, kvx.Batch([], [], [0], s.pages), s.normal(1, 4, 64), 4, 0.1, s.normal(1, 4, 64))


def test_streams_and_capture(setup):  # noqa: F811
    s = setup([300, 0, 17], [40, 2, 1], 2, 64, kvx.KVX_KV_FP8_PAGE, cross=True)
    held = s.fill(lens=s.P)
    q, want, _ = run(s, held, 2, 0.125)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = torch.empty_like(q)
    kvx.cross_attention(s.pool, s.batch, q, 4, 0.125, out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out.zero_()
        with pytest.raises(kvx.KvxError) as e:
            kvx.cross_attention(s.pool, s.batch, q, 4, 0.125, out, stream=side)
        assert e.value.status == kvx.KVX_EUNSUPPORTED


def test_encoder_and_decoder_together(setup):  # noqa: F811
    """A decoder's step: self attention on a pool of its own, cross attention to the encoder's states."""
    L, hist = [150, 61], [20, 33]
    for dtype in POOLS:
        enc = setup(L, [1, 1], 4, 64, dtype, cross=True)
        dec = setup(hist, [1, 1], 4, 64, dtype, seed=1)
        states, own = enc.fill(lens=L), dec.fill()
        q = dec.normal(2, 4, 64)
        x, y = torch.empty_like(q), torch.empty_like(q)
        kvx.extend_attention(dec.pool, dec.batch, q, 4, 0.125, x)
        kvx.cross_attention(enc.pool, enc.batch, x, 4, 0.125, y)
        for r in range(2):
            o, _, to, _ = ref.attend(ref.f64(q[r:r + 1]), *own[r], 0.125)
            ref.check(ref.f64(x[r:r + 1]), o, to, "self")
            o, _, to, _ = ref.attend(ref.f64(x[r:r + 1]), *states[r], 0.125)
            ref.check(ref.f64(y[r:r + 1]), o, to, "cross")
