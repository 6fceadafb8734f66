"""treewy_cache_append against a 64-bit reference: what is written, that nothing else is, lengths and flags."""
import numpy as np
import pytest
import torch

from tests.hybrid_reference import BF, F32, angles, rotate64, trees
from paper_2608_20961_amd import workload as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hy():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_20961_amd import hybrid
    return hybrid


def setup(seed, B, H, N, d, page, lens, dtype, width, tokens_major=True):
    g = torch.Generator().manual_seed(seed)
    n_pages = B * width + 2
    kp, vp = (torch.randn(n_pages, H, page, d, generator=g).to(dtype) for _ in range(2))
    table = torch.randperm(n_pages, generator=g)[:B * width].reshape(B, width).int()
    shape = (B, N, H, d) if tokens_major else (B, H, N, d)
    k, v = (torch.randn(shape, generator=g).to(dtype) for _ in range(2))
    if tokens_major:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    return k, v, kp, vp, table, torch.tensor(lens, dtype=torch.int32)


def expect(k, v, kp, vp, table, lens, cos, sin, nodes):
    """Pages after the call in 64 bits, and where they were written; nodes: what each sequence appends."""
    K, V = kp.double(), vp.double()
    hit = torch.zeros(kp.shape[0], kp.shape[2], dtype=torch.bool)
    page = kp.shape[2]
    for b, at in enumerate(nodes):
        pos = int(lens[b]) + torch.arange(len(at))
        kr = rotate64(k[b][:, at], pos, cos, sin)
        for l, p in enumerate(pos.tolist()):
            i = int(table[b, p // page])
            K[i, :, p % page], V[i, :, p % page] = kr[:, l], v[b][:, at[l]].double()
            hit[i, p % page] = True
    return K, V, hit


def check(kp, vp, K, V, hit, old_k, rot):
    """Values, keys that do not rotate and all other rows to the bit; rotated keys to one rounding of the type (a bf16: half
    of 2^-7, and fp32's own errors; fp32: three roundings of parts that are at most |a| + |b|)."""
    assert torch.equal(vp.double(), V)
    assert torch.equal(kp[..., rot:].double(), K[..., rot:])
    miss = ~hit[:, None, :, None].expand(kp.shape)
    assert torch.equal(kp[miss], old_k[miss])
    if rot == 0:
        return
    big = K[..., :rot].abs().amax(-1, keepdim=True) * 2
    tol = (2.0 ** -8 * K[..., :rot].abs() if kp.dtype == BF else 0) + 2.0 ** -22 * big
    assert bool(((kp[..., :rot].double() - K[..., :rot]).abs() <= tol).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,rot,H,page", [(64, 16, 1, 8), (64, 64, 3, 16), (128, 0, 2, 32), (128, 32, 8, 64), (256, 64, 2, 16),
                                          (256, 256, 1, 128)])
@pytest.mark.parametrize("N", [1, 13, 131])
def test_tokens(hy, dtype, d, rot, H, page, N):
    B = 3
    lens, count = [0, page - 1, 5 * page + 3], [N, (N + 1) // 2, 0]
    width = -(-(5 * page + 3 + N) // page)
    x = k, v, kp, vp, table, len_ = setup(N + d, B, H, N, d, page, lens, dtype, width)
    cos, sin = angles(5 * page + 3 + N, rot)
    K, V, hit = expect(*x, cos, sin, [list(range(c)) for c in count])
    dev = lambda t: None if t is None else t.cuda()
    gk, gv, err = kp.cuda(), vp.cuda(), torch.zeros(B, dtype=torch.int32, device="cuda")
    new = hy.treewy_cache_append(dev(k), dev(v), gk, gv, dev(table), dev(len_), cos=dev(cos), sin=dev(sin),
                                 count=torch.tensor(count, dtype=torch.int32).cuda(), err=err)
    assert new.tolist() == [a + b for a, b in zip(lens, count)] and err.tolist() == [0] * B
    check(gk.cpu(), gv.cpu(), K, V, hit, kp, rot)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,L", [(2, 1), (16, 6), (256, 256)])
def test_paths(hy, dtype, N, L):
    B, H, d, page, rot = 5, 2, 128, 16, 64
    par = trees(N, B, N, L)
    rng = np.random.default_rng(N)
    nodes = [wl.ancestors_and_self(par[b], int(rng.integers(N))) for b in range(B - 1)] + [[]]
    path = np.full((B, L), -1, dtype=np.int32)
    for b, p in enumerate(nodes):
        path[b, :len(p)] = p
    lens = [0, 15, 16, 100, 40]
    width = -(-(100 + L) // page)
    x = k, v, kp, vp, table, len_ = setup(N, B, H, N, d, page, lens, dtype, width, tokens_major=False)
    cos, sin = angles(100 + L, rot)
    K, V, hit = expect(*x, cos, sin, nodes)
    gk, gv = kp.cuda(), vp.cuda()
    new = hy.treewy_cache_append(k.cuda(), v.cuda(), gk, gv, table.cuda(), len_.cuda(), cos=cos.cuda(), sin=sin.cuda(),
                                 path=torch.from_numpy(path).cuda(),
                                 count=torch.tensor([len(p) for p in nodes], dtype=torch.int32).cuda())
    assert new.tolist() == [a + len(p) for a, p in zip(lens, nodes)]
    check(gk.cpu(), gv.cpu(), K, V, hit, kp, rot)


def test_flags_leave_the_cache(hy):
    """A path that is not one, counts out of range, no room, positions past the table: nothing is written; a bad page: its
    tokens are not, the others are."""
    B, H, N, d, page, width = 8, 2, 6, 64, 8, 3
    lens = [3, 3, 3, 20, -1, 4, 4, 16]
    k, v, kp, vp, table, len_ = setup(1, B, H, N, d, page, lens, BF, width)
    table[6, 1] = kp.shape[0]
    path = torch.tensor([[0, 2, 2, -1], [0, 6, -1, -1], [1, 3, 5, -1], [0, 1, 2, 3], [0, 1, -1, -1], [0, 1, 2, -1],
                         [0, 1, 2, 4], [0, 1, 2, 3]], dtype=torch.int32)
    count = torch.tensor([3, 2, 5, 4, 2, -1, 4, 4], dtype=torch.int32)
    count[3] = 4                                                       # 20 + 4 = 24 fits the pages, not the 22 positions
    cos, sin = angles(22, 16)
    nodes = [[], [], [], [], [], [], [0, 1, 2, 4], [0, 1, 2, 3]]
    table_ok = table.clone()
    table_ok[6, 1] = 0
    K, V, hit = expect(k, v, kp, vp, table_ok, len_, cos, sin, [[]] * 6 + [[0, 1, 2, 4], [0, 1, 2, 3]])
    gk, gv, err = kp.cuda(), vp.cuda(), torch.zeros(B, dtype=torch.int32, device="cuda")
    new = hy.treewy_cache_append(k.cuda(), v.cuda(), gk, gv, table.cuda(), len_.cuda(), cos=cos.cuda(), sin=sin.cuda(),
                                 path=path.cuda(), count=count.cuda(), err=err)
    assert err.tolist() == [2, 2, 2, 8, 8, 2, 0, 0]
    assert new.tolist() == [3, 3, 3, 20, -1, 4, 8, 20]
    check(gk.cpu(), gv.cpu(), K, V, hit, kp, 16)
    table[6, 0] = -1                                                   # now the page that holds positions 4 to 7
    gk, gv = kp.cuda(), vp.cuda()
    hy.treewy_cache_append(k.cuda(), v.cuda(), gk, gv, table.cuda(), len_.cuda(), cos=cos.cuda(), sin=sin.cuda(),
                           path=path.cuda(), count=count.cuda(), err=err.zero_())
    assert err.tolist() == [2, 2, 2, 8, 8, 2, 4, 0] and len(nodes) == B
    K, V, hit = expect(k, v, kp, vp, table_ok, len_, cos, sin, [[]] * 7 + [[0, 1, 2, 3]])
    check(gk.cpu(), gv.cpu(), K, V, hit, kp, 16)


def test_pages_past_four_gibibytes(hy):
    """Offsets in a cache of 5 GiB of keys: the first and the last page."""
    H, page, d = 8, 64, 256
    n_pages = 5 * 2 ** 30 // (H * page * d * 2)
    kp, vp = (torch.zeros(n_pages, H, page, d, dtype=BF, device="cuda") for _ in range(2))
    table = torch.tensor([[0, n_pages - 1]], dtype=torch.int32, device="cuda")
    k, v = (torch.randn(1, H, page + 5, d, device="cuda").to(BF) for _ in range(2))
    new = hy.treewy_cache_append(k, v, kp, vp, table, torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert new.tolist() == [page + 5]
    for p, x in ((kp, k), (vp, v)):
        assert torch.equal(p[0], x[0, :, :page]) and torch.equal(p[-1, :, :5], x[0, :, page:])
        assert not bool(p[1:-1].any()) and not bool(p[-1, :, 5:].any())
