"""treewy_tree_attention against a 64-bit reference.

Tolerances, normwise per (sequence, head) as everywhere here: bf16 rounds q and the draft's k (2^-9 each, relative), which moves
a score of size s by some 2^-9 s, the likelihoods (2^-9) and o (2^-9); scores here reach about 6, so that a result is off by
less than 2e-2 of the slice's largest; fp32 sums of d products and of all keys, and 2^y to an ulp: below 2e-5."""
import math

import numpy as np
import pytest
import torch

from tests.gpu_harness import rel_err, say
from tests.hybrid_reference import BF, F32, Context, angles, attention64, trees

pytestmark = pytest.mark.gpu

TOL = {BF: 2e-2, F32: 2e-5}


@pytest.fixture(scope="module")
def hy():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_20961_amd import hybrid
    return hybrid


def draft(seed, B, Hq, H, N, d, dtype):
    """q, k, v as parts of one projection's output [B, N, heads, d]."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, N, Hq + 2 * H, d, generator=g).to(dtype)
    return [t.transpose(1, 2) for t in (x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:])]


def gpu_views(q, k, v):
    return [t.transpose(1, 2).cuda().transpose(1, 2) for t in (q, k, v)]


def compare(o, ref, dtype):
    o = o.float().cpu().numpy()
    worst = max(rel_err(o[b, h], ref[b, h].numpy()) for b in range(ref.shape[0]) for h in range(ref.shape[1]))
    assert worst <= TOL[dtype], worst
    return worst


def run(hy, seed, lens, Hq, H, N, d, page, dtype, rot, parents, shared=0, scale=None, told=None):
    B = len(lens)
    q, k, v = draft(seed, B, Hq, H, N, d, dtype)
    ctx = Context(seed, lens, H, d, page, dtype, shared=shared)
    cos, sin = angles(max(lens) + N, rot)
    par = None if parents is None else torch.from_numpy(parents).int().cuda()
    err = torch.zeros(B, dtype=torch.int32, device="cuda")
    dev = lambda t: None if t is None else t.cuda()
    o = hy.treewy_tree_attention(*gpu_views(q, k, v), par, *ctx.gpu(), cos=dev(cos), sin=dev(sin),
                                 shared_len=shared if told is None else told, scale=scale, err=err)
    assert err.tolist() == [0] * B
    e = compare(o, attention64(q, k, v, parents, ctx, cos, sin, scale), dtype)
    say("[gpu] attention %s: %.1e" % ((lens, Hq, H, N, d, page), e))
    return o


LENS = [0, 1, 31, 32, 33, 64, 127, 128, 129, 300]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,rot,Hq,H,page", [(64, 16, 4, 4, 8), (64, 64, 7, 1, 32), (128, 128, 8, 2, 64), (128, 0, 32, 2, 16),
                                             (256, 64, 16, 2, 16), (256, 256, 2, 2, 128)])
@pytest.mark.parametrize("N", [1, 5])
def test_short_drafts(hy, dtype, d, rot, Hq, H, page, N):
    par = trees(N + d, len(LENS), N)
    run(hy, d + N, LENS, Hq, H, N, d, page, dtype, rot, par)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,Hq,H", [(64, 6, 2), (128, 8, 2), (256, 8, 1)])
@pytest.mark.parametrize("N", [17, 64, 100])
def test_wide_trees(hy, dtype, d, Hq, H, N):
    run(hy, d + N, [0, 65, 200], Hq, H, N, d, 16, dtype, d // 4, trees(N, 3, N))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,N", [(64, 256), (128, 256), (256, 200)])
def test_chunks_of_a_prompt(hy, dtype, d, N):
    """Chains without a parent array, and the same with one, bit for bit."""
    lens = [0, 77]
    a = run(hy, N, lens, 2, 1, N, d, 32, dtype, d, None)
    b = run(hy, N, lens, 2, 1, N, d, 32, dtype, d, np.tile(np.arange(-1, N - 1), (2, 1)))
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,Hq,H,N,B", [(128, 8, 2, 1, 3), (128, 8, 2, 1, 40), (256, 16, 2, 2, 5), (64, 4, 4, 9, 6)])
def test_shared_prefix(hy, dtype, d, Hq, H, N, B):
    rng = np.random.default_rng(B)
    shared = 203
    lens = [int(x) for x in rng.integers(shared, 2 * shared, B)]
    lens[0], lens[1] = 40, shared                                     # shorter than the shared part, and just it
    run(hy, B + d, lens, Hq, H, N, d, 16, dtype, 32, trees(B, B, N), shared=shared)
    run(hy, B + d, lens, Hq, H, N, d, 16, dtype, 32, trees(B, B, N), shared=shared, told=64)
    run(hy, B + d, lens, Hq, H, N, d, 16, dtype, 32, None, shared=shared, told=0)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,Hq,H,N,B", [(128, 8, 8, 1, 20), (128, 32, 8, 8, 20), (256, 32, 4, 2, 24), (64, 16, 16, 3, 30),
                                          (64, 16, 16, 32, 20)])
def test_shared_prefix_of_many(hy, dtype, d, Hq, H, N, B):
    """Enough shared keys that reading them once pays; sequences that end inside them and with them."""
    rng = np.random.default_rng(B)
    shared = 1100
    lens = [int(x) for x in rng.integers(shared, shared + 200, B)]
    lens[0], lens[1], lens[2] = 40, shared, 1024
    for told in (shared, 1024, 5000):
        if told == 5000:
            lens = [shared - 50] * B
        run(hy, B + d, lens, Hq, H, N, d, 32, dtype, 32, trees(B, B, N), shared=shared, told=min(told, max(lens)))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_bad_page_among_the_shared(hy, dtype):
    """Its keys are left out for every sequence, which are all told; as without shared_len."""
    B, H, d, shared = 20, 8, 128, 1024
    lens = [shared + 30 * b for b in range(B)]
    lens[3] = 60
    q, k, v = draft(5, B, H, H, 1, d, dtype)
    ctx = Context(5, lens, H, d, 32, dtype, shared=shared)
    kp, vp, table, cached = ctx.gpu()
    table[:, 7] = kp.shape[0] + 9
    table[3, 7] = 0
    out = []
    for told in (0, shared):
        err = torch.zeros(B, dtype=torch.int32, device="cuda")
        out.append(hy.treewy_tree_attention(*gpu_views(q, k, v), None, kp, vp, table, cached, shared_len=told, err=err))
        assert err.tolist() == [0 if b == 3 else 4 for b in range(B)]
    compare(out[1], out[0].double().cpu(), dtype)


def test_shared_longer_than_any(hy):
    run(hy, 3, [50, 50, 0], 4, 1, 1, 128, 16, BF, 0, None, shared=50, told=5000)


@pytest.mark.parametrize("B,ctx", [(1, 20000), (3, 9001), (300, 40)])
def test_long_and_many(hy, B, ctx):
    """One long sequence over many workgroups, ragged ones, and more sequences than a wave has lanes."""
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, ctx + 1, B)]
    lens[-1] = ctx
    run(hy, B, lens, 4, 1, 1, 128, 64, BF, 128, None)


@pytest.mark.parametrize("d,Hq,H,N", [(64, 6, 2, 100), (64, 8, 1, 40), (128, 8, 2, 90), (128, 2, 1, 129), (256, 16, 2, 17),
                                      (256, 16, 2, 64), (256, 3, 1, 100)])
@pytest.mark.parametrize("rot", [16, 64])
def test_wide_table(hy, d, Hq, H, N, rot):
    """A table as wide as a long context's, of which little is in use: the kernels for much work."""
    lens = [0, 65, 500, 1]
    q, k, v = draft(d + N, 4, Hq, H, N, d, BF)
    ctx = Context(N, lens, H, d, 32, BF)
    cos, sin = angles(max(lens) + N, rot)
    par = trees(N, 4, N)
    kp, vp, table, cached = ctx.gpu()
    wide = torch.full((4, 30000), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    err = torch.zeros(4, dtype=torch.int32, device="cuda")
    o = hy.treewy_tree_attention(*gpu_views(q, k, v), torch.from_numpy(par).int().cuda(), kp, vp, wide, cached, cos=cos.cuda(),
                                 sin=sin.cuda(), err=err)
    assert err.tolist() == [0] * 4
    e = compare(o, attention64(q, k, v, par, ctx, cos, sin, None), BF)
    say("[gpu] attention, wide table %s: %.1e" % ((Hq, H, N, d, rot), e))


def test_enough_units_for_one_each(hy):
    run(hy, 8, [int(x) for x in np.random.default_rng(8).integers(0, 90, 200)], 8, 8, 2, 64, 16, BF, 32, None)


@pytest.mark.parametrize("B,H,N,d", [(64, 4, 1, 256), (87, 3, 3, 256), (64, 8, 1, 64), (131, 4, 2, 128), (500, 2, 1, 64),
                                     (40, 8, 70, 128), (520, 1, 1, 64)])
@pytest.mark.parametrize("kind", ["equal", "ragged", "one long", "none"])
def test_units_whole_or_in_parts(hy, B, H, N, d, kind):
    """About as many (sequence, head)s as workgroups: whole, or cut where one is longer than the rest together."""
    lens = {"equal": [64] * B, "ragged": [int(x) for x in np.random.default_rng(B).integers(0, 400, B)],
            "one long": [3] * (B // 2) + [9000] + [5] * (B - B // 2 - 1), "none": [0] * B}[kind]
    o = run(hy, B + d, lens, H, H, N, d, 16, BF, 32, trees(B, B, N))
    assert torch.equal(o, run(hy, B + d, lens, H, H, N, d, 16, BF, 32, trees(B, B, N)))


@pytest.mark.parametrize("scale", [-0.1, 0.0, 1.7])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_scales(hy, scale, dtype):
    run(hy, 5, [0, 70], 4, 2, 6, 64, 16, dtype, 16, trees(5, 2, 6), scale=scale)


def test_large_scores(hy):
    """Scores in the thousands, of both signs: only the largest counts."""
    q, k, v = draft(9, 2, 2, 1, 3, 64, F32)
    ctx = Context(9, [150, 0], 1, 64, 16, F32)
    par = trees(9, 2, 3)
    o = hy.treewy_tree_attention(*gpu_views(1000 * q, k, v), torch.from_numpy(par).int().cuda(), *ctx.gpu(), scale=1.0)
    ref = attention64(1000 * q, k, v, par, ctx, None, None, 1.0)
    # (a score of some 1e4 is off by 64 products' roundings: up to 1e4 x 2^-24 x 8, which moves a likelihood by as much)
    assert max(rel_err(o[b, h].cpu().numpy(), ref[b, h].numpy()) for b in range(2) for h in range(2)) <= 2e-2


@pytest.mark.parametrize("dtype", [BF, F32])
def test_what_a_node_does_not_see_cannot_matter(hy, dtype):
    """Infinities and NaNs in the keys and values of nodes off the path change no other node's bits; where they are seen the
    result is not finite.  (The context's unused rows and pages hold NaNs in every test here.)"""
    B, N, Hq, H, d = 2, 40, 4, 2, 128
    par = trees(11, B, N, 8)
    q, k, v = draft(11, B, Hq, H, N, d, dtype)
    ctx = Context(11, [100, 0], H, d, 16, dtype)
    P = torch.from_numpy(par).int().cuda()
    a = hy.treewy_tree_attention(*gpu_views(q, k, v), P, *ctx.gpu())
    bad = [5, 23, 39]
    k, v = k.clone(), v.clone()
    k[:, :, bad[0]], v[:, :, bad[0]] = math.nan, math.nan
    v[:, :, bad[1], 7] = math.inf
    v[:, :, bad[2]], k[:, :, bad[2]] = -math.inf, math.inf
    b = hy.treewy_tree_attention(*gpu_views(q, k, v), P, *ctx.gpu())
    for s in range(B):
        hit = np.zeros(N, dtype=bool)
        for t in range(N):
            hit[t] = t in bad or (par[s, t] >= 0 and hit[par[s, t]])
        clean = torch.from_numpy(~hit).cuda()
        assert torch.equal(a[s][:, clean], b[s][:, clean])
        for t in np.flatnonzero(hit):
            assert not bool(torch.isfinite(b[s, :, t]).all()), t
    assert bool(torch.isfinite(a).all())


def test_flags(hy):
    B, N, H, d, page = 5, 4, 1, 64, 8
    q, k, v = draft(13, B, 2, H, N, d, F32)
    ctx = Context(13, [20, 20, 20, 20, 20], H, d, page, F32)
    par = np.tile(np.array([-1, 0, 1, 1]), (B, 1))
    broken = par.copy()
    broken[1, 2] = 3                                                   # counts as -1
    kp, vp, table, lens = ctx.gpu()
    table[2, 1] = ctx.n_pages + 5                                      # tokens 8 to 15 are left out
    lens[3], lens[4] = -7, 1000                                        # count as 0, and as all that the table holds
    table[4] = table[0, 0]
    err = torch.zeros(B, dtype=torch.int32, device="cuda")
    o = hy.treewy_tree_attention(*gpu_views(q, k, v), torch.from_numpy(broken).int().cuda(), kp, vp, table, lens, err=err)
    assert err.tolist() == [0, 1, 4, 8, 8]
    par[1, 2] = -1
    width = table.shape[1]
    ctx.K[2], ctx.V[2] = (torch.cat([x[:, :8], x[:, 16:]], 1) for x in (ctx.K[2], ctx.V[2]))
    ctx.K[3], ctx.V[3] = (x[:, :0] for x in (ctx.K[3], ctx.V[3]))
    ctx.K[4], ctx.V[4] = (x[:, :8].repeat(1, width, 1) for x in (ctx.K[0], ctx.V[0]))
    ctx.lens = [20, 20, 12, 0, 8 * width]
    compare(o, attention64(q, k, v, par, ctx, None, None), F32)
    cos, sin = (x.cuda() for x in angles(21, 16))                      # positions 21 to 23 take the last row's angles
    err.zero_()
    hy.treewy_tree_attention(*gpu_views(q, k, v), torch.from_numpy(par).int().cuda(), *ctx_gpu_plain(13), cos=cos, sin=sin, err=err)
    assert err.tolist() == [8] * B


def ctx_gpu_plain(seed):
    return Context(seed, [20] * 5, 1, 64, 8, F32).gpu()


def test_layouts_streams_and_repeats(hy):
    """Heads-first, tokens-first and padded rows, outputs of every layout, a workspace of the caller's, another stream, and
    fresh inputs in between: the same bits."""
    B, N, Hq, H, d = 3, 9, 8, 2, 128
    q, k, v = (t.cuda() for t in draft(17, B, Hq, H, N, d, BF))
    ctx = Context(17, [500, 33, 260], H, d, 16, BF).gpu()
    par = torch.from_numpy(trees(17, B, N)).int().cuda()
    cos, sin = (x.cuda() for x in angles(600, 64))
    call = lambda *x, **kw: hy.treewy_tree_attention(*x, par, *ctx, cos=cos, sin=sin, **kw)
    a = call(q.contiguous(), k.contiguous(), v.contiguous())
    pad = torch.zeros(B, N, Hq + 2, d + 8, dtype=BF, device="cuda")
    pad[:, :, :Hq, :d] = q.transpose(1, 2)
    o = torch.zeros(B, N, Hq, d, dtype=BF, device="cuda").transpose(1, 2)
    need = hy.lib.treewy_tree_attention_workspace(0, N, B, Hq, H, d, 1)
    r = call(pad[:, :, :Hq, :d].transpose(1, 2), k, v, o=o, workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda"))
    assert r is o and torch.equal(a, o)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = call(q, k, v, stream=side)
    side.synchronize()
    assert torch.equal(a, b)
    for _ in range(3):
        call(torch.randn_like(q), k, v)
        assert torch.equal(a, call(q, k, v))
    with pytest.raises(hy.TreewyError):
        call(q, k, v, workspace=torch.empty(need - 16, dtype=torch.uint8, device="cuda"))


def test_replayed_graph(hy):
    """Captured once, replayed with other lengths, trees and inputs, eager work in between."""
    B, N, Hq, H, d = 4, 6, 8, 2, 128
    ctx = Context(19, [700, 33, 260, 5], H, d, 16, BF).gpu()
    s = dict(q=torch.zeros(B, Hq, N, d, dtype=BF, device="cuda"), k=torch.zeros(B, H, N, d, dtype=BF, device="cuda"),
             v=torch.zeros(B, H, N, d, dtype=BF, device="cuda"), par=torch.zeros(B, N, dtype=torch.int32, device="cuda"),
             o=torch.zeros(B, Hq, N, d, dtype=BF, device="cuda"), lens=ctx[3].clone())
    ws = torch.empty(hy.lib.treewy_tree_attention_workspace(0, N, B, Hq, H, d, 1), dtype=torch.uint8, device="cuda")
    call = lambda o: hy.treewy_tree_attention(s["q"], s["k"], s["v"], s["par"], *ctx[:3], s["lens"], o=o, workspace=ws)
    call(s["o"])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(s["o"])
    for i in range(4):
        for n in ("q", "k", "v"):
            s[n].copy_(torch.randn(s[n].shape, device="cuda"))
        s["par"].copy_(torch.from_numpy(trees(20 + i, B, N)))
        s["lens"].copy_((ctx[3].float() * (0.2 * (i + 1))).int())
        g.replay()
        torch.cuda.synchronize()
        got = s["o"].clone()
        assert torch.equal(got, call(torch.empty_like(got)))


def test_cache_past_four_gibibytes(hy):
    H, page, d, N = 8, 64, 256, 1
    n_pages = 5 * 2 ** 30 // (H * page * d * 2)
    kp, vp = (torch.empty(n_pages, H, page, d, dtype=BF, device="cuda") for _ in range(2))
    at = [n_pages - 1, 0, n_pages // 2, n_pages - 2]
    ctx = Context(23, [230], H, d, page, BF, spare=0)
    for i, p in enumerate(at):
        src = int(ctx.table[0, i])
        kp[p], vp[p] = ctx.k[src].cuda(), ctx.v[src].cuda()
    q, k, v = draft(23, 1, 8, H, N, d, BF)
    o = hy.treewy_tree_attention(*gpu_views(q, k, v), None, kp, vp, torch.tensor([at], dtype=torch.int32, device="cuda"),
                                 torch.tensor([230], dtype=torch.int32, device="cuda"))
    compare(o, attention64(q, k, v, None, ctx, None, None), BF)
