"""Attention where magnitudes lie far apart: values of the cache many binades below others of the same
call, whether a row sees those or not.  And each of its kernels: every number of blocks of channels and of
column tiles.  Against plain 64-bit forms.

Bounds, beside those of the attention tests: a value is exact whatever else the cache holds, so an
output's error is relative to what its row sees of its channel.  A key whose weight is below 2^-160 of
its row's largest has none in float32 (a weight is at most 2^16 times 2^-160 of that, below its least
2^-126), so it brings no error either.
"""
import numpy as np
import pytest
import torch

import attn_ref as R
from paper_2204_03418_amd import coinf
from test_gpu_attn import WEIGHT, attend_case, attend_check, make_pages
from test_gpu_tokens import BF16, DEV, F32, U, gen, randn

pytestmark = pytest.mark.gpu


def attend_seen(q, k, v, pos, window, scale):
    """One stream's values and sizes as attn_ref.attend's, with a reach of the keys that have a weight."""
    y, (size, worst, reach) = R.attend(q, k, v, pos, 0, window, scale)
    g = q.shape[1] // k.shape[1]
    for t in range(len(q)):
        a = max(0, pos[t] - window + 1 if window else 0)
        kk, vv = (np.repeat(x[a:pos[t] + 1], g, 1) for x in (k, v))
        s = scale * (kk * q[t]).sum(-1)
        some = s - s.max(0) > -160 * np.log(2.0)
        reach[t] = np.abs(vv * some[..., None]).sum(0)
    return y, (size, worst, reach)


def far_values(kind, v, ctx, T, window):
    """v (B, L, K, D) with magnitudes far apart."""
    L = v.shape[1]
    x = torch.zeros(L)                                          # binades a token
    if kind == "blocks":                                        # channels 0..31, 32..63, ..
        step = torch.tensor([60.0, 0.0, -60.0, -100.0, 30.0, -30.0, 50.0, -90.0])
        return v * torch.exp2(step[torch.arange(v.shape[-1]) // 32])
    if kind == "later":                                         # half of the newest see no large one
        x[ctx + (T + 1) // 2:] = 45
    elif kind == "far later":
        x[:] = -70
        x[ctx + (T + 1) // 2:] = 90
    elif kind == "left":                                        # in the window's tile, out of it
        x[:max(ctx + 1 - window, 0)] = 50
    elif kind == "growing":
        x = torch.arange(L) * (160.0 / L) - 80
    elif kind == "falling":
        x = 80 - torch.arange(L) * (160.0 / L)
    elif kind == "zeros first":
        x[:] = 70
        v = v.clone()
        v[:, :L // 2] = 0
    elif kind == "tiny":
        x[:] = -110
    elif kind == "one block":                                   # one token, one block, far up
        v = v.clone()
        v[:, 5, :, :32] *= 2.0 ** 60
        return v
    return v * torch.exp2(x)[:, None, None]


KINDS = ["blocks", "later", "far later", "left", "growing", "falling", "zeros first", "tiny",
         "one block"]


def far_case(kind, T, ctx, H, K, D, dtype, window, P=16, B=2):
    """A layer that holds ctx tokens and the newest T's outputs, and what they are within."""
    g = gen(101)
    q = randn(g, B, T, H, D, dtype=dtype)
    k = randn(g, B, ctx + T, K, D, dtype=dtype)
    v = far_values(kind, randn(g, B, ctx + T, K, D), ctx, T, window).to(dtype)
    W = -(-(ctx + T) // P) + 1
    pages = make_pages(B, B * W, W, P, K, D)
    attn = coinf.CoAttention(pages, heads=H, window=window or None, dtype=dtype)
    if ctx:
        pages.reserve(ctx)
        attn.append(k[:, :ctx].to(DEV), v[:, :ctx].to(DEV))
    pages.reserve(T)
    got = attn.forward_steps(q.to(DEV), k[:, ctx:].to(DEV), v[:, ctx:].to(DEV))
    kq, vq = R.quantised(R.np64(k)), R.quantised(R.np64(v))
    pos = ctx + np.arange(T)
    for b in range(B):
        y, sizes = attend_seen(R.np64(q[b]), kq[b], vq[b], pos, window, attn.scale)
        keys = min(ctx + T, window or 1 << 30)
        bound = R.attend_bound(y, sizes, keys, D, U[dtype], WEIGHT[dtype])
        R.within(got[b], y, bound, f"{kind} stream {b}")
    return attn, q, got


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,ctx,H,K,D", [
    (80, 70, 4, 2, 64), (40, 0, 2, 1, 96), (150, 200, 2, 1, 40), (70, 100, 2, 2, 128),
    (36, 90, 1, 1, 256)])
def test_many_rows(kind, dtype, T, ctx, H, K, D):
    far_case(kind, T, ctx, H, K, D, dtype, 60 if kind == "left" else 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["growing", "later"])
@pytest.mark.parametrize("D", [32, 64, 96, 128])
def test_wide_workgroups(D, kind, dtype):
    """More than 128 rows over 8192 keys and more: workgroups of 256 rows."""
    far_case(kind, 140, 8300, 1, 1, D, dtype, 0, P=64, B=1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,ctx,H,K,D", [
    (1, 70, 4, 4, 64), (4, 70, 4, 2, 64), (6, 130, 4, 1, 96), (1, 1500, 8, 2, 128), (3, 40, 2, 1, 40),
    (2, 90, 2, 2, 256), (1, 60, 2, 1, 16)])
def test_few_rows(kind, dtype, T, ctx, H, K, D):
    far_case(kind, T, ctx, H, K, D, dtype, 60 if kind == "left" else 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [2, 6, 90])
def test_masked_values_do_not_change_rows(dtype, T):
    """Later tokens' values 2^20 times larger, for bfloat16: earlier rows keep every bit, since the
    values stay exact 16-bit floats.  By more, and for float32, where these blocks' own scales (2^3
    apart) pass the 2^21 that stay normal 16-bit floats: they stay within what the weights'
    roundings (twice, of either call) may change."""
    g = gen(102)
    B, H, K, D, ctx = 2, 4, 2, 64, 50
    q, k = randn(g, B, T, H, D, dtype=dtype), randn(g, B, ctx + T, K, D, dtype=dtype)
    v = randn(g, B, ctx + T, K, D, dtype=dtype)
    half = T // 2
    outs = {}
    for up in (0, 20, 60, 120):
        w = v.clone()
        w[:, ctx + half:] *= 2.0 ** up
        pages = make_pages(B, 24, 12, 16, K, D)
        attn = coinf.CoAttention(pages, heads=H, dtype=dtype)
        pages.reserve(ctx)
        attn.append(k[:, :ctx].to(DEV), w[:, :ctx].to(DEV))
        pages.reserve(T)
        y = attn.forward_steps(q.to(DEV), k[:, ctx:].to(DEV), w[:, ctx:].to(DEV))
        outs[up] = y[:, :half].double()
    if dtype is BF16:
        assert torch.equal(outs[0], outs[20])
    _, vq = (R.quantised(R.np64(x)) for x in (k, v))
    # |y| <= max |v|; a rounding of either, the weights of either, sums of at most ctx + T terms
    most = torch.from_numpy(np.abs(vq).max(1)).to(DEV)[:, None].repeat_interleave(H // K, 2)
    room = most * (2 * U[dtype] + 4 * WEIGHT[dtype] + 2 * (ctx + T + 64) * R.U32
                   + 4 * (D + 16) * R.U32 * 100)
    for up in (20, 60, 120):
        assert ((outs[up] - outs[0]).abs() <= room).all(), up


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [1, 40])
def test_a_key_without_weight(dtype, T):
    """A token that every row sees with a weight of exp(-1000) and less, whose values are 2^100 times
    the others': as if it were not there."""
    g = gen(103)
    B, H, K, D, ctx = 2, 2, 1, 64, 40
    q, k = randn(g, B, T, H, D, dtype=dtype), randn(g, B, ctx + T, K, D, dtype=dtype)
    v = randn(g, B, ctx + T, K, D, dtype=dtype)
    q[..., 0] = 8
    k[..., 0] = 0
    k[:, 5] = 0
    k[:, 5, :, 0] = -2000
    v[:, 5] *= 2.0 ** 100
    pages = make_pages(B, 24, 12, 16, K, D)
    attn = coinf.CoAttention(pages, heads=H, dtype=dtype)
    pages.reserve(ctx)
    attn.append(k[:, :ctx].to(DEV), v[:, :ctx].to(DEV))
    pages.reserve(T)
    got = attn.forward_steps(q.to(DEV), k[:, ctx:].to(DEV), v[:, ctx:].to(DEV))
    kq, vq = R.quantised(R.np64(k)), R.quantised(R.np64(v))
    for b in range(B):
        y, (size, worst, reach) = attend_seen(R.np64(q[b]), kq[b], vq[b], ctx + np.arange(T), 0,
                                              attn.scale)
        assert np.abs(y).max() < 100
        # the magnitudes of the scores that count
        kk = kq[b].copy()
        kk[5] = 0
        _, (_, worst, _) = R.attend(R.np64(q[b]), kk, vq[b], ctx + np.arange(T), 0, 0, attn.scale)
        bound = R.attend_bound(y, (size, worst, reach), ctx + T, D, U[dtype], WEIGHT[dtype])
        R.within(got[b], y, bound, f"stream {b}")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_prompts_and_tokens_agree(dtype):
    """A prompt's outputs and those of the same tokens one at a time, the later values 2^45 larger."""
    g = gen(104)
    B, T, H, K, D = 2, 50, 4, 2, 64
    q, k, v = (randn(g, B, T, n, D, dtype=dtype) for n in (H, K, K))
    v[:, T // 2:] *= 2.0 ** 45
    pages = make_pages(B, 16, 8, 16, K, D)
    attn = coinf.CoAttention(pages, heads=H, dtype=dtype)
    prompt = attn.forward(q.to(DEV), k.to(DEV), v.to(DEV))
    one = []
    for t in range(T):
        pages.reserve(1)
        one.append(attn.forward_step(*(x[:, t].contiguous().to(DEV) for x in (q, k, v))))
    kq, vq = R.quantised(R.np64(k)), R.quantised(R.np64(v))
    for b in range(B):
        y, sizes = R.attend(R.np64(q[b]), kq[b], vq[b], np.arange(T), 0, 0, attn.scale)
        bound = R.attend_bound(y, sizes, T, D, U[dtype], WEIGHT[dtype])
        for got, what in ((prompt, "prompt"), (torch.stack(one, 1), "tokens")):
            R.within(got[b], y, bound, f"{what} stream {b}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [2, 80])
def test_what_is_not_finite_beside_far_values(dtype, T):
    """A value block that is not finite reaches who sees it, the far values around it nobody else."""
    g = gen(105)
    B, H, K, D, ctx, at = 2, 2, 1, 96, 30, 12
    q, k, v = (randn(g, B, L, n, D, dtype=dtype) for L, n in ((T, H), (ctx + T, K), (ctx + T, K)))
    v = far_values("growing", v.float(), ctx, T, 0).to(dtype)
    outs = []
    for bad in (True, False):
        w = v.clone()
        if bad:
            w[0, at, 0, 40] = float("inf")
        pages = make_pages(B, 24, 12, 16, K, D)
        attn = coinf.CoAttention(pages, heads=H, dtype=dtype)
        pages.reserve(ctx)
        attn.append(k[:, :ctx].to(DEV), w[:, :ctx].to(DEV))
        pages.reserve(T)
        outs.append(attn.forward_steps(q.to(DEV), k[:, ctx:].to(DEV), w[:, ctx:].to(DEV)))
    hit = torch.zeros_like(outs[0], dtype=torch.bool)
    hit[0, ..., 32:64] = True
    assert torch.isnan(outs[0][hit]).all()
    assert torch.equal(outs[0][~hit], outs[1][~hit]) and torch.isfinite(outs[1]).all()


def test_far_values_in_a_graph():
    """A captured call whose values come to lie far apart between replays."""
    g = gen(106)
    B, T, H, K, D = 2, 40, 2, 1, 64
    q, k = (randn(g, B, T, n, D, dtype=BF16).to(DEV) for n in (H, K))
    v = randn(g, B, T, K, D, dtype=BF16).to(DEV)
    pages = make_pages(B, 8, 4, 16, K, D)
    attn = coinf.CoAttention(pages, heads=H, dtype=BF16)
    pages.reserve(T)
    buf = v.clone()
    attn.forward_steps(q, k, buf)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = attn.forward_steps(q, k, buf)
    for up in (0, 60, 0, 110):
        buf.copy_(v)
        buf[:, T // 2:] *= 2.0 ** up
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, attn.forward_steps(q, k, buf)), up


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("up", [10, 13, 16])
@pytest.mark.parametrize("T,D", [(1, 64), (6, 96), (90, 64), (40, 256)])
def test_queries_with_an_outlier(dtype, up, T, D):
    """A query channel 2^up times the others whose keys are 0: the scores are the others'.

    bfloat16: a block's queries are two terms of 4 bits whose least step is 2^-9 and 2^-13 of a scale
    that is at most 2^-7 of the block's largest, so what they leave is half of 2^-13 2^-7 of that,
    2^-21, for each of the block's keys."""
    g = gen(107)
    B, H, K, ctx = 2, 2, 1, 60
    q, k, v = (randn(g, B, L, n, D, dtype=dtype) for L, n in ((T, H), (ctx + T, K), (ctx + T, K)))
    q[..., 3] = 2.0 ** up * 1.5
    k[..., 3] = 0
    pages = make_pages(B, 24, 12, 16, K, D)
    attn = coinf.CoAttention(pages, heads=H, dtype=dtype)
    pages.reserve(ctx)
    attn.append(k[:, :ctx].to(DEV), v[:, :ctx].to(DEV))
    pages.reserve(T)
    got = attn.forward_steps(q.to(DEV), k[:, ctx:].to(DEV), v[:, ctx:].to(DEV))
    kq, vq = R.quantised(R.np64(k)), R.quantised(R.np64(v))
    for b in range(B):
        qb = R.np64(q[b])
        y, (size, worst, reach) = R.attend(qb, kq[b], vq[b], ctx + np.arange(T), 0, 0, attn.scale)
        if dtype is BF16:
            left = 0
            for c in range(0, D, 32):
                keys = np.abs(kq[b][..., c:c + 32]).sum(-1).max()
                left = left + 2.0 ** -21 * np.abs(qb[..., c:c + 32]).max(-1, keepdims=True) * keys
            worst = worst + attn.scale * left / ((D + 16) * R.U32)
        bound = R.attend_bound(y, (size, worst, reach), ctx + T, D, U[dtype], WEIGHT[dtype])
        R.within(got[b], y, bound, f"stream {b}")


# ------------------------------------------------------------ every kernel of attention

HEADS = [24, 40, 96, 128, 160, 192, 224, 256]                   # 1 to 8 blocks of channels


@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("T,H,K,rows", [(1, 1, 1, 1), (4, 8, 2, 16), (3, 12, 2, 18), (8, 4, 1, 32)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", HEADS)
def test_few_rows_of_every_head(D, dtype, T, H, K, rows, P):
    """One and two column tiles of 16 rows, over a context of several parts."""
    assert T * H // K == rows <= 32                             # the kernel of few rows
    case = (2, T, 1300, H, K, D, P, 0, dtype, "full", 0, 0)
    attn, pages, q, *rest = attend_case(case, 33)
    attend_check(case, attn, q, *rest, attn.attend(q.to(DEV)), "few rows")


@pytest.mark.parametrize("T,ctx,H,K", [(20, 700, 2, 1), (70, 100, 2, 1)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", HEADS)
def test_many_rows_of_every_head(D, dtype, T, ctx, H, K):
    assert T * H // K > 32                                      # the kernel of many rows
    case = (2, T, ctx, H, K, D, 32, 0, dtype, "ragged", 0, 0)
    attn, pages, q, *rest = attend_case(case, 34)
    attend_check(case, attn, q, *rest, attn.attend(q.to(DEV)), "many rows")


@pytest.mark.parametrize("kind", ["blocks", "growing"])
@pytest.mark.parametrize("T,H,K", [(1, 1, 1), (4, 6, 1), (40, 1, 1)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", HEADS)
def test_far_values_of_every_head(D, dtype, T, H, K, kind):
    far_case(kind, T, 150, H, K, D, dtype, 0, P=32, B=1)


def test_rotary_writes_queries_and_keys_apart():
    """One tensor may be both inputs; two outputs may not be one place."""
    layer = coinf.CoRotary(32, device=DEV)
    x = randn(gen(108), 2, 3, 4, 32).to(DEV)
    a, b = layer.forward(x, x)
    assert torch.equal(a, b) and torch.equal(a, layer.forward(x))
    other = x.clone()
    for k, out, k_out in ((other, x, x), (other, other, None), (other, None, x)):
        with pytest.raises(coinf.CoinfError):
            layer.forward(x, k, out=out, k_out=k_out)
