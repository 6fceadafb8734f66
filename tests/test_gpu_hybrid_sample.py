"""treewy_sample: the token equals the definition's (whole-number likelihoods, from the device's 2^y) on every row, and lies
where 64 bits put the drawn point, up to 2e-5 of the sum (2^y and y in float32 are off by less than 4e-6, relative, where a
likelihood counts; top_p's boundary moves with them)."""
import math

import numpy as np
import pytest
import torch

from tests.gpu_harness import say
from tests.hybrid_reference import BF, F32, kept64

pytestmark = pytest.mark.gpu
EPS = 2e-5


@pytest.fixture(scope="module")
def hy():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_20961_amd import hybrid
    return hybrid


def share(W, x):
    f = (x.clamp(0.0, 1.0) * 2.0 ** 31).long()
    return (W >> 31) * f + (((W & (2 ** 31 - 1)) * f) >> 31)


def definition(logits, u, temperature, top_k=None, top_p=None, min_p=None):
    x = logits.float()
    R, V = x.shape
    x = torch.where(torch.isnan(x), -math.inf, x)
    top = x.amax(-1, keepdim=True)
    t = torch.ones(R, device="cuda") if temperature is None else temperature
    greedy = ~(t > 0)
    slope = torch.full_like(t, math.log2(math.e)) / torch.where(greedy, 1.0, t)
    y = torch.where(x == top, 0.0, x - top) * slope[:, None]
    w = torch.where(x == -math.inf, 0, (torch.exp2(y) * 2.0 ** 40).long())
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    rank = torch.arange(V, device="cuda").expand(R, V)
    if min_p is not None:
        ws = torch.where(ws >= (torch.nan_to_num(min_p).clamp(0, 1) * 2.0 ** 40).long()[:, None], ws, 0)
    k = torch.full((R,), V, device="cuda") if top_k is None else torch.where(top_k > 0, top_k, V)
    k = torch.where(greedy, 1, k)
    ws = torch.where(rank < k[:, None], ws, 0)
    if top_p is not None:
        off = ~(top_p < 1)
        most = share(ws.sum(-1), torch.where(off, 1.0, top_p))
        ws = torch.where((ws.cumsum(-1) - ws < most[:, None]) | (rank == 0) | off[:, None], ws, 0)
    kept = torch.zeros_like(w).scatter_(1, order, ws)
    at = share(kept.sum(-1), torch.nan_to_num(u).clamp(0.0, 1.0 - 2.0 ** -24))
    token = (kept.cumsum(-1) <= at[:, None]).sum(-1)
    return torch.where(top[:, 0] == -math.inf, -1, token).int()


def logits_of(g, R, V, dtype, kind):
    if kind == "flat":
        x = 0.3 * torch.randn(R, V, generator=g, device="cuda")
    elif kind == "ties":
        x = torch.randint(-3, 4, (R, V), generator=g, device="cuda").float()
    elif kind == "peaked":
        x = 3.0 * torch.randn(R, V, generator=g, device="cuda")
        x.scatter_(1, torch.randint(0, V, (R, min(V, 30)), generator=g, device="cuda"), 9 + 3 * torch.randn(R, min(V, 30), generator=g, device="cuda"))
    else:                                                              # masked by a grammar: most tokens impossible
        x = 3.0 * torch.randn(R, V, generator=g, device="cuda")
        x[torch.rand(R, V, generator=g, device="cuda") < 0.97] = -math.inf
        x[:, V // 2] = 1.0
    return x.to(dtype)


def filters(g, R, mode):
    p = dict(temperature=0.3 + 1.5 * torch.rand(R, generator=g, device="cuda"))
    if mode in ("topk", "all"):
        p["top_k"] = torch.randint(0, 300, (R,), generator=g, device="cuda", dtype=torch.int32)
    if mode in ("topp", "all"):
        p["top_p"] = 0.2 + 0.9 * torch.rand(R, generator=g, device="cuda")
    if mode in ("minp", "all"):
        p["min_p"] = 0.3 * torch.rand(R, generator=g, device="cuda") ** 3
    return p


def near(x, u, token, p):
    """Whether 64 bits allow the token: it holds the drawn point, up to EPS, for a top_p up to EPS away."""
    for f in (1.0, 1 - EPS, 1 + EPS):
        top_p = p.get("top_p")
        w = kept64(x, p["temperature"], p.get("top_k"), None if top_p is None else top_p * f, p.get("min_p"))
        c = np.cumsum(w) / w.sum()
        if w[token] > 0 and c[token] - w[token] / w.sum() - EPS <= u <= c[token] + EPS:
            return True, math.log(w[token] / w.sum())
    return False, 0.0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [1, 2, 63, 513, 8192, 32001, 150000])
@pytest.mark.parametrize("kind", ["flat", "ties", "peaked", "masked"])
def test_every_filter(hy, dtype, V, kind):
    for i, mode in enumerate(("plain", "topk", "topp", "minp", "all")):
        g = torch.Generator(device="cuda").manual_seed(1000 * i + V)
        R = 24
        x, u, p = logits_of(g, R, V, dtype, kind), torch.rand(R, generator=g, device="cuda"), filters(g, R, mode)
        err = torch.zeros(R, dtype=torch.int32, device="cuda")
        token, lp = hy.treewy_sample(x, u, err=err, **p)
        assert err.tolist() == [0] * R
        ref = definition(x, u, **p)
        assert torch.equal(token, ref), (mode, (token != ref).nonzero().flatten().tolist())
        rows = range(0, R, 6)
        for r in rows:
            ok, want = near(x[r].float().cpu().numpy(), float(u[r]), int(token[r]), {n: float(v[r]) if n != "top_k" else int(v[r]) for n, v in p.items()})
            assert ok, (mode, r)
            assert abs(float(lp[r]) - want) <= 1e-4 + 2 * EPS * abs(want), (mode, r)


def test_edges(hy):
    """Rows with nothing, infinities, NaNs, both zeros, zero temperature, filters at and past their ends, u at its ends."""
    inf, nan = math.inf, math.nan
    rows = [([-inf] * 4, {}), ([nan] * 4, {}), ([nan, 1, nan, 1], {}), ([inf, 0, inf, -inf], {}), ([0.0, -0.0, 0.0, -1], dict(top_k=2)),
            ([1, 3, 3, 2], dict(temperature=0.0)), ([1, 3, 3, 2], dict(temperature=-1.0)), ([1, 3, 3, 2], dict(temperature=nan)),
            ([1, 3, 3, 2], dict(temperature=inf)), ([1, 3, -inf, 2], dict(temperature=inf)), ([1, 3, 3, 2], dict(temperature=1e-30)),
            ([1, 3, 3, 2], dict(top_p=0.0)), ([1, 3, 3, 2], dict(top_p=-1.0)), ([1, 3, 3, 2], dict(top_p=nan)),
            ([1, 3, 3, 2], dict(top_p=1.0)), ([1, 3, 3, 2], dict(min_p=1.0)), ([1, 3, 3, 2], dict(min_p=7.0)),
            ([1, 3, 3, 2], dict(min_p=nan)), ([1, 3, 3, 2], dict(top_k=1)), ([1, 3, 3, 2], dict(top_k=4)),
            ([1, 3, 3, 2], dict(top_k=-3)), ([-1e38, -3e38, -1e38, -2e38], {}), ([3e38, -3e38, 0, 3e38], {})]
    for u in (0.0, 0.3, 0.9999999, 1.0, -2.0, nan):
        R = len(rows)
        x = torch.tensor([r for r, _ in rows], device="cuda")
        col = lambda n, d, t=torch.float32: torch.tensor([p.get(n, d) for _, p in rows], device="cuda", dtype=t)
        p = dict(temperature=col("temperature", 1.0), top_k=col("top_k", 0, torch.int32), top_p=col("top_p", 1.0), min_p=col("min_p", 0.0))
        err = torch.zeros(R, dtype=torch.int32, device="cuda")
        U = torch.full((R,), u, device="cuda")
        token, lp = hy.treewy_sample(x, U, err=err, **p)
        q = dict(p, temperature=torch.where(torch.isinf(p["temperature"]), 1e30, p["temperature"]))
        assert token.tolist() == definition(x, U, **q).tolist(), u
        assert err.tolist() == [16, 16] + [0] * (R - 2) and lp[:2].tolist() == [-inf] * 2
        assert bool((lp[2:] <= 0).all()) and token[5:8].tolist() == [1, 1, 1] and lp[5:8].tolist() == [0.0] * 3
        assert int(token[11]) == int(token[12]) == 1                  # the first of the largest


def test_frequencies(hy):
    """u on an even grid: every token comes as often as its likelihood says, to one draw."""
    V, n = 37, 20000
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(V, generator=g, device="cuda")
    u = (torch.arange(n, device="cuda") + 0.5) / n
    token, _ = hy.treewy_sample(x.expand(n, V), u, temperature=torch.full((n,), 0.8, device="cuda"),
                                top_k=torch.full((n,), 20, device="cuda", dtype=torch.int32))
    w = kept64(x.cpu().numpy(), 0.8, 20, None, None)
    assert np.abs(np.bincount(token.cpu().numpy(), minlength=V) - n * w / w.sum()).max() <= 1.5


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strided_rows_streams_and_repeats(hy, dtype):
    """Rows at any distance and alignment, another stream, no logprob left behind, repeats: the same bits."""
    g = torch.Generator(device="cuda").manual_seed(5)
    R, V = 9, 1001
    wide = torch.randn(R, V + 30, generator=g, device="cuda").to(dtype)
    u = torch.rand(R, generator=g, device="cuda")
    p = filters(g, R, "all")
    for start in (0, 1, 3, 8):
        x = wide[:, start:start + V]
        token, lp = hy.treewy_sample(x, u, **p)
        assert torch.equal(token, definition(x, u, **p))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        t2, l2 = hy.treewy_sample(x.contiguous(), u, stream=side, **p)
        side.synchronize()
        assert torch.equal(token, t2) and torch.equal(lp, l2)
    back = wide.flip(0)[:, :V]
    assert torch.equal(hy.treewy_sample(back, u, **p)[0], definition(back, u, **p))
    say("[gpu] sample rows at every alignment")


def test_the_devices_exponential(hy):
    """The definition's 2^y is the device's: what torch's exp2 gives for every y of the range, to the bit, or these tests would
    compare the kernel with something else."""
    n = 1 << 22
    x = -40.0 * torch.rand(n // 64, 64, device="cuda")
    x[:, 0] = 0.0
    u = torch.rand(n // 64, device="cuda")
    assert torch.equal(hy.treewy_sample(x, u)[0], definition(x, u, None))
