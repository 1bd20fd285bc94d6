"""GPU parity of the page and row movements of the cache (kv_reserve, kv_release,
kv_fork, kv_append, kv_prune) with the oracle: tables, counts, lengths and cache
bytes are equal, untouched bytes included."""
import numpy as np
import pytest
import torch

from oracle import serving as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dreams():
    import paper_2606_00535_gb300 as d
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    d._lib()
    return d


def i32(v):
    return torch.tensor(np.asarray(v, dtype=np.int32), device="cuda")


class Pool:
    """A pool on both sides: numpy arrays and the framework's tensors."""

    def __init__(self, dreams, B, P, pages, layers=1, Hkv=1, D=8, seed=0, table=None, ref=None):
        rng = np.random.default_rng(seed)
        self.d, self.rng = dreams, rng
        self.k, self.v = (rng.integers(0, 1 << 15, (layers, pages, 64, Hkv, D)).astype(np.int16) for _ in range(2))
        self.table = np.full((B, P), -1, np.int32) if table is None else np.asarray(table, np.int32)
        self.ref = np.zeros(pages, np.int32) if ref is None else np.asarray(ref, np.int32)
        self.gk, self.gv = (torch.from_numpy(x).view(torch.bfloat16).cuda() for x in (self.k, self.v))
        self.gt, self.gr = i32(self.table), i32(self.ref)
        self.kv = dreams.KVCache(self.gk, self.gv, self.gt)
        self.pool = dreams.PagePool(self.kv, self.gr)
        self.st = torch.zeros(1, dtype=torch.int32, device="cuda")

    def same(self, flags=0):
        torch.cuda.synchronize()
        assert int(self.st.item()) == flags
        self.st.zero_()
        np.testing.assert_array_equal(self.gt.cpu().numpy(), self.table)
        np.testing.assert_array_equal(self.gr.cpu().numpy(), self.ref)
        for a, b in ((self.gk, self.k), (self.gv, self.v)):
            assert np.array_equal(a.view(torch.int16).cpu().numpy(), b)

    def reserve(self, lens, n):
        self.d.kv_reserve(self.pool, i32(lens), i32(n), status=self.st)
        self.table, self.ref, f = S.reserve(self.table, self.ref, lens, n)
        self.same(f)
        return f

    def release(self, begin, end):
        self.d.kv_release(self.pool, i32(begin), i32(end), status=self.st)
        self.table, self.ref, f = S.release(self.table, self.ref, begin, end)
        self.same(f)
        return f

    def fork(self, parent, lens, alias=False):
        g = i32(lens)
        new = self.d.kv_fork(self.pool, i32(parent), g, new_kv_len=g if alias else None, status=self.st)
        self.table, self.ref, lens, f = S.fork(self.table, self.ref, parent, lens, [self.k, self.v])
        self.same(f)
        np.testing.assert_array_equal(new.cpu().numpy(), lens)
        return lens, f

    def append(self, lens, n, T_max, layer=0, fused=3):
        B, (_, _, _, H, D) = len(lens), self.k.shape
        x = self.rng.integers(0, 1 << 15, (B, T_max, fused, H, D)).astype(np.int16)
        g = torch.from_numpy(x).view(torch.bfloat16).cuda()
        self.d.kv_append(self.kv, g[:, :, 0], g[:, :, fused - 1], i32(lens), i32(n), layer=layer, status=self.st)
        f = 0
        for b in range(B):
            if n[b] < 0 or n[b] > T_max or lens[b] < 0 or lens[b] + n[b] > self.table.shape[1] * 64:
                f |= S.BAD_KV_LEN
                continue
            for t in range(n[b]):
                pg = self.table[b, (lens[b] + t) // 64]
                if not 0 <= pg < len(self.ref):
                    f |= S.BAD_PAGE
                    continue
                self.k[layer, pg, (lens[b] + t) % 64] = x[b, t, 0]
                self.v[layer, pg, (lens[b] + t) % 64] = x[b, t, fused - 1]
        self.same(f)


@pytest.mark.parametrize("B,P,pages", [(1, 1, 1), (3, 5, 12), (70, 9, 500), (2000, 3, 5000)])
def test_reserve_and_release(dreams, B, P, pages):
    p = Pool(dreams, B, P, pages, seed=B)
    rng = p.rng
    lens = np.zeros(B, np.int32)
    for _ in range(5):
        n = rng.integers(0, 64 * P - lens + 1).astype(np.int32) // 2
        f = p.reserve(lens, n)
        lens = np.where([all(p.table[b, : -(-(lens[b] + n[b]) // 64)] >= 0) for b in range(B)], lens + n, lens).astype(np.int32)
        p.release(np.full(B, 3), lens - 70)      # behind a window
        p.release(lens, np.full(B, P * 64))      # the unused tail
        keep = rng.random(B) < 0.7
        p.release(np.zeros(B), np.where(keep, 0, P * 64))
        lens = np.where(keep, lens, 0).astype(np.int32)


def test_reserve_scans_a_large_pool(dreams):
    """Free pages in the last places of a pool larger than one pass of the scan."""
    pages = 20011
    ref = np.ones(pages, np.int32)
    ref[[5, 4095, 4096, 9000, 20009, 20010]] = 0
    p = Pool(dreams, 2, 4, pages, ref=ref)
    assert p.reserve([0, 0], [64 * 4, 65]) == 0
    assert p.table.tolist() == [[5, 4095, 4096, 9000], [20009, 20010, -1, -1]]


def test_reserve_refusals(dreams):
    """Too few pages: rows in order until one does not fit; bad lengths and
    entries and shared pages skip their row alone."""
    p = Pool(dreams, 5, 4, 8, ref=[0, 0, 1, 0, 0, 0, 2, 1], table=[[-1] * 4, [2, -1, -1, -1], [6, -1, -1, -1], [-1] * 4, [7, -1, -1, -1]])
    f = p.reserve([0, 10, 20, 0, 64], [128, 100, 100, 200, 1])
    assert f == dreams.DATA_NO_PAGES | dreams.DATA_SHARED_PAGE
    p = Pool(dreams, 4, 2, 8, ref=[1] + [0] * 7, table=[[-1, -1], [99, -1], [-2, -1], [0, -1]])
    assert p.reserve([0, 0, 0, 0], [129, 80, 80, 80]) == dreams.DATA_BAD_KV_LEN | dreams.DATA_BAD_PAGE
    assert p.table[3, 1] == 1
    assert p.reserve([-1, 0, 0, 0], [1, -5, 0, 0]) == dreams.DATA_BAD_KV_LEN
    assert p.release([-1, 0, 0, 0], [64, 129, 0, 0]) == dreams.DATA_BAD_KV_LEN
    assert p.release([0, 0, 0, 0], [0, 64, 128, 128]) == dreams.DATA_BAD_PAGE


@pytest.mark.parametrize("B,P,layers,Hkv,D", [(2, 2, 1, 1, 8), (8, 4, 3, 2, 64), (40, 6, 2, 3, 128), (1100, 2, 1, 1, 8)])
def test_forks(dreams, B, P, layers, Hkv, D):
    p = Pool(dreams, B, P, B * P + 2, layers, Hkv, D, seed=B)
    rng = p.rng
    lens = rng.integers(0, 64 * P + 1, B).astype(np.int32)
    lens[0], lens[1] = 64 * (P - 1) + 1, 64
    p.reserve(np.zeros(B, np.int32), lens)
    for kind in ("best", "draw", "rotate", "some", "self"):
        parent = {"best": np.zeros(B), "draw": rng.integers(0, B, B), "rotate": (np.arange(B) + 1) % B,
                  "some": rng.integers(-1, B, B), "self": np.arange(B)}[kind].astype(np.int32)
        lens, f = p.fork(parent, lens, alias=kind in ("draw", "rotate"))
        assert f == 0
        grow = np.minimum(64 * P - lens, rng.integers(0, 50, B)).astype(np.int32)
        if p.reserve(lens, grow) == 0:
            p.append(lens, grow, 64, layer=layers - 1)
            lens = lens + grow


def test_fork_refusals_change_nothing(dreams):
    p = Pool(dreams, 3, 2, 5)
    p.reserve([0, 0, 0], [100, 64, 30])
    before = p.table.copy()
    assert p.fork([0, 0, 0], [100, 64, 30])[1] == 0  # two free, and two let go
    p = Pool(dreams, 3, 2, 4)
    p.reserve([0, 0, 0], [100, 64, 30])
    before = p.table.copy()
    assert p.fork([0, 0, 1], [100, 64, 30])[1] == 0
    p = Pool(dreams, 3, 1, 3)
    p.reserve([0, 0, 0], [10, 10, 10])
    before = p.table.copy()
    p2 = Pool(dreams, 4, 1, 3, table=[[0], [1], [2], [-1]], ref=[1, 1, 1])
    assert p2.fork([0, 1, 2, 0], [10, 10, 10, 0])[1] == dreams.DATA_NO_PAGES
    assert p.fork([0, 3, 0], [10, 10, 10])[1] == dreams.DATA_BAD_INDEX
    assert p.fork([0, -2, 0], [10, 10, 10])[1] == dreams.DATA_BAD_INDEX
    assert p.fork([0, 1, 0], [10, 65, 10])[1] == dreams.DATA_BAD_KV_LEN
    assert p.fork([0, 1, 0], [10, -1, 10])[1] == dreams.DATA_BAD_KV_LEN
    np.testing.assert_array_equal(p.table, before)
    p.table[2, 0] = -1
    p.gt[2, 0] = -1
    assert p.fork([0, 1, 2], [10, 10, 10])[1] == dreams.DATA_BAD_PAGE
    p.table[2, 0] = 3
    p.gt[2, 0] = 3
    assert p.fork([0, 1, 0], [10, 10, 10])[1] == dreams.DATA_BAD_PAGE


@pytest.mark.parametrize("Hkv,D,T", [(1, 8, 1), (4, 128, 1), (8, 64, 77), (5, 64, 200)])
def test_append_paged(dreams, Hkv, D, T):
    p = Pool(dreams, 4, 5, 30, 2, Hkv, D, seed=T)
    lens, n = np.array([0, 63, 64, 100]), np.array([T, max(0, T - 3), T, 0])
    p.reserve(lens, n)
    for layer in (0, 1):
        p.append(lens, n, T, layer)
    p.append([0, -1, 10, 64 * 5 - 1], [T + 1, 0, -1, 2], T)                     # bad lengths
    q = Pool(dreams, 2, 5, 30, 1, Hkv, D, table=[[3, -1, 4, -1, -1], [77, 5, 6, 7, 8]])
    q.append([0, 0], [min(T, 130), 1], T)                                       # pages missing


def test_append_contiguous_and_dense_rows(dreams):
    g = torch.Generator().manual_seed(1)
    k = torch.randn((3, 100, 2, 64), generator=g).to(torch.bfloat16)
    new = torch.randn((2, 3, 7, 2, 64), generator=g).to(torch.bfloat16)
    kv = dreams.KVCache(k.cuda(), k.clone().cuda())
    dreams.kv_append(kv, new[0].cuda(), new[1].cuda(), i32([0, 93, 50]), i32([7, 7, 2]))
    for x, y in ((kv.k, new[0]), (kv.v, new[1])):
        ref = k.clone()
        ref[0, :7], ref[1, 93:], ref[2, 50:52] = y[0], y[1], y[2, :2]
        assert torch.equal(x.cpu(), ref)
    # one token of one sequence, from an expanded (stride 0) batch dimension
    one = new[:1, 0, :1].cuda()
    dreams.kv_append(dreams.KVCache(kv.k[:1].contiguous(), kv.v[:1].contiguous()), one, one, i32([5]), i32([1]))


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("layers,B,Hkv,D,v0,n_vis,r,text", [
    (1, 1, 1, 8, 0, 1, 1, 1), (1, 2, 4, 128, 17, 300, 150, 200), (3, 3, 2, 64, 5, 700, 1, 90), (2, 1, 32, 128, 64, 128, 127, 600),
    (1, 1, 3, 8, 0, 500, 0, 3), (40, 2, 8, 128, 35, 100, 50, 77), (2, 2, 5, 64, 1, 64, 64, 9), (2, 2, 5, 64, 1, 0, 0, 9)])
def test_prune(dreams, paged, layers, B, Hkv, D, v0, n_vis, r, text):
    rng = np.random.default_rng(r)
    L = v0 + n_vis + text
    P = -(-L // 64)
    lens = np.array([L - i * (text // (2 * B)) for i in range(B)], np.int32)
    keep = np.stack([np.sort(rng.choice(n_vis, r, replace=False)) + v0 if r else np.zeros(0, int) for _ in range(B)]).astype(np.int32)
    table = rng.permutation(B * P).reshape(B, P).astype(np.int32)
    k, v = (rng.integers(0, 1 << 15, (layers, B * P, 64, Hkv, D)).astype(np.int16) for _ in range(2))
    if not paged:
        table = np.arange(B * P).reshape(B, P)
    gk, gv = (torch.from_numpy(x).view(torch.bfloat16).cuda() for x in (k, v))
    shape = gk.shape if paged else (layers, B, P * 64, Hkv, D)
    kv = dreams.KVCache(gk.view(shape), gv.view(shape), i32(table) if paged else None)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ref = torch.ones(B * P, dtype=torch.int32, device="cuda") if paged else None
    new = dreams.kv_prune(kv, i32(keep).view(B, r), v0, n_vis, i32(lens), refcount=ref, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    np.testing.assert_array_equal(new.cpu().numpy(), lens - (n_vis - r))
    for x, g in ((k, gk), (v, gv)):
        y = x.copy()
        for b in range(B):
            for d, s in S.prune_moves(keep[b], v0, n_vis, lens[b]):
                y[:, table[b, d // 64], d % 64] = x[:, table[b, s // 64], s % 64]
        assert np.array_equal(g.view(torch.int16).cpu().numpy(), y)


def test_prune_refusals(dreams):
    """Each bad sequence is left alone; the one good sequence is pruned."""
    rng = np.random.default_rng(9)
    B, P, n_vis, r = 7, 4, 100, 40
    k = rng.integers(0, 1 << 15, (1, B * P, 64, 1, 8)).astype(np.int16)
    table = np.arange(B * P).reshape(B, P).astype(np.int32)
    keep = np.stack([np.sort(rng.choice(n_vis, r, replace=False)) + 3 for _ in range(B)]).astype(np.int32)
    lens = np.full(B, 200, np.int32)
    keep[1, 7] = keep[1, 6]
    keep[2, r - 1] = 103
    lens[3], lens[4] = 102, 257
    table[5, 2] = -1
    ref = np.ones(B * P, np.int32)
    ref[table[6, 1]] = 2
    gk = torch.from_numpy(k).view(torch.bfloat16).cuda()
    gv = gk.clone()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    new = dreams.kv_prune(dreams.KVCache(gk, gv, i32(table)), i32(keep), 3, n_vis, i32(lens), refcount=i32(ref), status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == (dreams.DATA_BAD_INDEX | dreams.DATA_BAD_KV_LEN | dreams.DATA_BAD_PAGE | dreams.DATA_SHARED_PAGE)
    assert new.cpu().tolist() == [140] + lens[1:].tolist()
    y = k.copy()
    for d, s in S.prune_moves(keep[0], 3, n_vis, 200):
        y[:, table[0, d // 64], d % 64] = k[:, table[0, s // 64], s % 64]
    assert np.array_equal(gk.view(torch.int16).cpu().numpy(), y) and np.array_equal(gv.view(torch.int16).cpu().numpy(), y)


def test_fork_past_32_bit_offsets(dreams):
    """A page whose elements start past 2^32: 32-layer-sized strides in one layer."""
    Hkv, D = 8, 128
    pages = (1 << 32) // (64 * Hkv * D) + 4
    k = torch.zeros((pages, 64, Hkv, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    k[pages - 1], v[pages - 1] = 3.0, 4.0
    table = torch.full((2, 1), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = pages - 1
    ref = torch.ones(pages, dtype=torch.int32, device="cuda")
    ref[pages - 2] = 0
    pool = dreams.PagePool(dreams.KVCache(k, v, table), ref)
    new = dreams.kv_fork(pool, i32([0, 0]), i32([50, 0]))
    assert new.tolist() == [50, 50] and table.tolist() == [[pages - 1], [pages - 2]] and int(ref[pages - 2]) == 1
    assert (k[pages - 2, :50] == 3).all() and (v[pages - 2, :50] == 4).all() and (k[pages - 2, 50:] == 0).all()


@pytest.mark.parametrize("B,P", [(3000, 1), (200, 30), (2500, 2), (700, 60), (65535, 1)])
def test_forks_of_large_tables(dreams, B, P):
    """Tables of one CTA and of a cluster, with rows in shared memory and in the workspace, in one turn and in several."""
    p = Pool(dreams, B, P, B + B // 2 + 2 * P, seed=B + P)
    rng = p.rng
    # groups of rows share full pages; every row of a group has its own last page
    lens = np.zeros(B, np.int32)
    free = list(rng.permutation(B + B // 2 + 2 * P)[: B + 2 * P])
    shared = [free.pop() for _ in range(P)]
    for b in range(B):
        full = int(rng.integers(0, P))
        lens[b] = 64 * full + int(rng.integers(0, 64)) if free else 64 * full
        p.table[b, :full] = shared[:full]
        if lens[b] % 64:
            p.table[b, full] = free.pop()
    np.add.at(p.ref, p.table[p.table >= 0], 1)
    p.gt.copy_(i32(p.table)), p.gr.copy_(i32(p.ref))
    for parent in (rng.integers(-1, B, B), (np.arange(B) // 4) * 4 + rng.integers(0, 4, B), np.arange(B)[::-1]):
        parent = np.minimum(parent, B - 1).astype(np.int32)
        before = p.table.copy()
        new, f = p.fork(parent, lens)
        if f == 0:
            lens = new
        else:
            assert f == dreams.DATA_NO_PAGES
            np.testing.assert_array_equal(p.table, before)
    bad = np.arange(B)
    bad[B // 2] = B
    assert p.fork(bad, lens)[1] == dreams.DATA_BAD_INDEX
    full = np.flatnonzero(lens % 64)
    q = int(full[len(full) // 2])
    p.table[q, lens[q] // 64] = -1
    p.gt[q, int(lens[q]) // 64] = -1
    assert p.fork(np.arange(B), lens)[1] == dreams.DATA_BAD_PAGE
    p.table[B - 1, P - 1] = p.gt[B - 1, P - 1] = len(p.ref)
    assert p.fork(np.arange(B), lens)[1] == dreams.DATA_BAD_PAGE


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("B,Hkv,D,v0,n_vis,r,text", [(1, 1, 8, 3, 20000, 9000, 70), (2, 1, 8, 130, 150000, 8193, 300), (1, 2, 16, 60, 9000, 8192, 140000),
                                                     (160, 4, 128, 1, 90, 30, 40), (1, 80, 128, 9, 300, 200, 60)])
def test_prune_long(dreams, paged, B, Hkv, D, v0, n_vis, r, text):
    """Lists and page tables that do not fit into shared memory; more walks than SMs; rows of more than one block."""
    test_prune(dreams, paged, 1, B, Hkv, D, v0, n_vis, r, text)


def test_reserve_many_rows(dreams):
    """Rows shared by 32 lanes down to one; more free pages wanted than shared memory holds."""
    for B, P in ((2, 70), (33, 40), (64, 9), (300, 20), (1025, 3), (5000, 2)):
        p = Pool(dreams, B, P, B * P + 7, seed=B)
        lens = np.zeros(B, np.int32)
        n = p.rng.integers(0, 64 * P + 1, B).astype(np.int32)
        n[B // 2], n[0] = 64 * P, 0
        lens[B // 3] = n[B // 3] // 2
        assert p.reserve(lens, n - lens) == 0
        p.release(np.full(B, 64), n - 64)
        p.reserve(np.zeros(B, np.int32), n)
