"""GPU: ancestor masks, accepted paths, moved rows, forked rows, block copies and shared
releases against plain lists; and whole decoding loops of them.  Integers have to be
equal, stored rows the same bits."""
import numpy as np
import pytest
import torch

from oracle import tree_ref
from oracle.tables_ref import release_ref
from paper_2507_08523_amd import ilpc, pipeline

pytestmark = pytest.mark.gpu

BLOCK = 16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a ROCm GPU (run with -m 'not gpu' on the CPU)")
    ilpc.load()
    yield
    torch.cuda.synchronize()


def dev(a, dtype=np.int32):
    return torch.from_numpy(np.array(a, dtype=dtype, order="C")).cuda()


def ints(t):
    return t.cpu().numpy().tolist()


def random_tree(n, rng, branch=2, pad=0.0):
    out = [-1] + [int(rng.integers(max(0, (i - 1) // branch - 2), (i - 1) // branch + 1)) for i in range(1, n)]
    for i in range(1, n):
        if rng.random() < pad:
            out[i] = int(rng.choice([-2, -1, i, i + 3, -(1 << 31), (1 << 31) - 1]))
    return out[:n]


def signed(words):
    return [w - (1 << 64) if w >> 63 else w for w in words]


# -- masks ------------------------------------------------------------------------

@pytest.mark.parametrize("sizes", [[1], [0], [64], [65], [5, 0, 64, 1, 63], [100, 128, 2], [200, 129, 256, 1], [1000, 30],
                                   [1024, 1023]])
@pytest.mark.parametrize("branch,pad", [(1, 0.0), (3, 0.0), (2, 0.2)])
def test_masks(sizes, branch, pad):
    rng = np.random.default_rng(sum(sizes) + branch)
    par = [random_tree(n, rng, branch, pad) for n in sizes]
    start = rng.integers(0, 5000, len(sizes))
    for extra_words in (0, 1):
        words = min(16, max(1, -(-max(sizes) // 64)) + extra_words)
        n = sum(sizes)
        masks, pos = dev(np.full((n + 3, words), 5), np.int64), dev([9] * (n + 3))
        cu = dev(np.concatenate([[0], np.cumsum(sizes)]))
        flat = dev(sum(par, []) + [0] * 3)
        ilpc.tree_masks(flat, cu, masks, pos, dev(start))
        only = dev(np.full((n + 3, words), 5), np.int64)
        ilpc.tree_masks(flat, cu, only)
        torch.cuda.synchronize()
        want_m, want_p = [], []
        for p, s in zip(par, start):
            m, q = tree_ref.masks_ref(p, int(s), words)
            want_m += [signed(x) for x in m]
            want_p += q
        assert ints(masks) == want_m + [[5] * words] * 3 and ints(pos) == want_p + [9] * 3
        assert torch.equal(only, masks)


def test_masks_of_a_chain_and_of_too_many_nodes():
    chain = list(range(-1, 149))
    for words in (1, 2, 3):
        m, p = dev(np.zeros((150, words)), np.int64), dev([0] * 150)
        ilpc.tree_masks(dev(chain), dev([0, 150]), m, p, dev([7]))
        torch.cuda.synchronize()
        wm, wp = tree_ref.masks_ref(chain, 7, words)
        assert ints(m) == [signed(x) for x in wm] and ints(p) == wp


def test_requests_with_rows_outside_the_buffers_are_taken_as_having_none():
    m, p = dev([[3]] * 6, np.int64), dev([9] * 6)
    ilpc.tree_masks(dev([-1, 0, 0, -1, 0, 1]), dev([0, 3, 7, 2, -1]), m, p)
    torch.cuda.synchronize()
    assert ints(m) == [[1], [3], [5], [3], [3], [3]] and ints(p) == [0, 1, 1, 9, 9, 9]


# -- accepted paths ------------------------------------------------------------------

def picks_for(par, tok, rng, hit=0.8, vocab=50):
    out = [int(x) for x in rng.integers(0, vocab, len(par))]
    for i in rng.permutation(len(par)):
        if 0 <= par[i] < i and rng.random() < hit:
            out[par[i]] = tok[i]
    return out


def run_accept(par, tok, pick, cu, start, root=None):
    n, B = len(par), len(start)
    outs = [dev([9] * n)] + [dev([9] * B) for _ in range(4)]
    ilpc.tree_accept(dev(par), dev(tok), dev(pick), dev(cu), dev(start), *outs,
                     root_targets=None if root is None else dev(root))
    torch.cuda.synchronize()
    return [ints(o) for o in outs]


@pytest.mark.parametrize("sizes", [[1], [0, 3], [64], [65, 1], [20] * 40, [300, 7, 256, 257], [1000]])
@pytest.mark.parametrize("branch,vocab,pad", [(1, 1000, 0.0), (3, 1000, 0.0), (2, 3, 0.0), (2, 20, 0.15)])
@pytest.mark.parametrize("rooted", [False, True])
def test_accept(sizes, branch, vocab, pad, rooted):
    rng = np.random.default_rng(sum(sizes) + vocab)
    par, tok, pick, path, rest = [], [], [], [], [[], [], [], []]
    start, root = rng.integers(0, 999, len(sizes)).tolist(), rng.integers(0, vocab, len(sizes)).tolist()
    for r, n in enumerate(sizes):
        p = random_tree(n, rng, branch, pad)
        t = rng.integers(0, vocab, n).tolist()
        k = picks_for(p, t, rng, vocab=vocab)
        if n and rng.random() < 0.7:
            root[r] = t[0]
        got, want = tree_ref.accept_ref(p, t, k, root[r] if rooted else None)
        par, tok, pick = par + p, tok + t, pick + k
        path += got + [-1] * (n - len(got))
        kept = start[r] + len(got)
        for o, x in zip(rest, (len(got), want, kept, -(-kept // 16))):
            o.append(x)
    cu = np.concatenate([[0], np.cumsum(sizes)])
    got = run_accept(par + [0, 0], tok + [0, 0], pick + [0, 0], cu, start, root if rooted else None)
    assert got == [path + [9, 9]] + rest


def test_a_long_chain_is_accepted_whole():
    n = 700
    tok = list(range(n))
    got = run_accept(list(range(-1, n - 1)), tok, tok[1:] + [5], [0, n], [16])
    assert got == [list(range(n)), [n], [5], [16 + n], [-(-(16 + n) // 16)]]


# -- moved rows -------------------------------------------------------------------

def pools(nb, Hkv, D, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    return rnd(nb, Hkv, 16, D), rnd(nb, Hkv, D, 16)


def same_bits(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("Hkv,D", [(1, 64), (8, 128), (3, 64), (2, 128)])
@pytest.mark.parametrize("sizes,counts", [([5], [5]), ([64], [7]), ([1, 0, 40, 20], [1, 0, 6, 0]), ([300, 33], [70, 33]),
                                          ([20] * 30, [4] * 30), ([1000], [400])])
def test_compact(Hkv, D, sizes, counts):
    rng = np.random.default_rng(sum(sizes) + D)
    start = rng.integers(0, 70, len(sizes))
    lens = start + sizes
    nb = int(sum(-(-lens // 16))) + 4
    ids = rng.permutation(nb)
    mb = int((-(-lens // 16)).max()) + 1
    bt, at = np.full((len(sizes), mb), -1), 0
    path = []
    for r, (n, k) in enumerate(zip(sizes, counts)):
        m = -(-int(lens[r]) // 16)
        bt[r, :m] = ids[at:at + m]
        at += m
        path += sorted(rng.choice(n, k, replace=False).tolist()) + [-1] * (n - k) if n else []
    kp, vp = pools(nb, Hkv, D)
    kp[0, 0, 0, 0], vp[1, 0, 0, 0] = float("nan"), float("inf")
    wk, wv = kp.clone(), vp.clone()
    cu = np.concatenate([[0], np.cumsum(sizes)])
    for r, k in enumerate(counts):
        s = start[r] + np.array(path[cu[r]:cu[r] + k], int)
        d = start[r] + np.arange(k)
        wk[bt[r, d // 16], :, d % 16] = kp[bt[r, s // 16], :, s % 16]
        wv[bt[r, d // 16], :, :, d % 16] = vp[bt[r, s // 16], :, :, s % 16]
    ilpc.kv_compact(kp, vp, dev(bt), dev(cu), dev(start), dev(path + [3]), dev(counts))
    torch.cuda.synchronize()
    assert same_bits(kp, wk) and same_bits(vp, wv)


def test_compact_leaves_out_what_is_not_there():
    kp, vp = pools(4, 2, 64)
    wk, wv = kp.clone(), vp.clone()
    # rows outside the path's range, blocks outside the pools, positions past the table, counts past the nodes
    bt, cu, start = dev([[0, 9, -1], [1, 2, -5], [3, 1 << 30, 3]]), dev([0, 20, 26, 29]), dev([14, 30, -4])
    path = np.full(29, -1)
    path[:3], path[20:26], path[26:29] = [1, 2, 99], [0, 1, 2, 3, 40, 5], [1, 2, 3]
    wk[0, :, 14], wv[0, :, :, 14] = kp[0, :, 15], vp[0, :, :, 15]  # the one move that is whole
    ilpc.kv_compact(kp, vp, bt, cu, start, dev(path), dev([3, 99, 3]))
    torch.cuda.synchronize()
    assert same_bits(kp, wk) and same_bits(vp, wv)


# -- copies, forks, releases ----------------------------------------------------------

def test_blocks_whose_offsets_pass_32_bits():
    nb, Hkv, D, n = 264000, 8, 128, 12  # 2^32 elements lie in the first 2^18 blocks
    big = [torch.empty(nb, Hkv, 16, D, dtype=torch.bfloat16, device="cuda"),
           torch.empty(nb, Hkv, D, 16, dtype=torch.bfloat16, device="cuda")]
    small = pools(2 * n, Hkv, D)
    ids = [nb - 1 - 37 * i for i in range(n)] + [131072 + i for i in range(n)]
    rows, at = dev([list(range(2 * n))]), torch.tensor(ids, device="cuda")
    for b, s in zip(big, small):
        b[at] = s
    P, nodes = 2 * n * 16 - 100, 60
    cu, start, path = dev([0, nodes]), dev([P]), dev([2 * i for i in range(30)] + [-1] * 30)
    masks = torch.zeros(nodes, 1, dtype=torch.int64, device="cuda")
    ilpc.tree_masks(dev(range(-1, nodes - 1)), cu, masks)
    for Hq in (8, 256, 512):  # of every kernel
        q = torch.randn(nodes, Hq, D, device="cuda").to(torch.bfloat16)
        outs = [torch.zeros_like(q) for _ in range(2)]
        for o, (kp, vp), table in zip(outs, (big, small), (dev([ids]), rows)):
            ilpc.paged_tree_attn(q, kp, vp, table, cu, dev([P + nodes]), nodes, D ** -0.5, masks, o)
        torch.cuda.synchronize()
        assert same_bits(*outs)
    for (kp, vp), table in ((big, dev([ids])), (small, rows)):
        ilpc.kv_compact(kp, vp, table, cu, start, path, dev([30]))
    ilpc.copy_blocks(*big, dev(ids[:3]), dev(ids[n + 3:n + 6]))
    ilpc.copy_blocks(*small, dev([0, 1, 2]), dev([n + 3, n + 4, n + 5]))
    torch.cuda.synchronize()
    assert all(same_bits(b[at], s) for b, s in zip(big, small))


@pytest.mark.parametrize("Hkv,D", [(1, 64), (8, 128), (3, 64), (32, 128)])
@pytest.mark.parametrize("n", [1, 2, 50])
def test_copy_blocks(Hkv, D, n):
    nb = 2 * n + 3
    kp, vp = pools(nb, Hkv, D)
    rng = np.random.default_rng(n)
    ids = rng.permutation(nb)
    src, dst = ids[:n].copy(), ids[n:2 * n].copy()
    src[n // 2:] = src[0]  # one block to several places
    bad = n > 2
    if bad:
        src[1], dst[3], src[5], dst[6] = -1, -1, nb, 1 << 30
    wk, wv = kp.clone(), vp.clone()
    for s, d in zip(src, dst):
        if 0 <= s < nb and 0 <= d < nb:
            wk[d], wv[d] = kp[s], vp[s]
    ilpc.copy_blocks(kp, vp, dev(src), dev(dst))
    torch.cuda.synchronize()
    assert same_bits(kp, wk) and same_bits(vp, wv)


class Rows:
    """A batch of rows, some of which hold requests, over `first` blocks of the cache and a free list."""

    def __init__(self, B, live, hi, first, spare, seed, width=None):
        rng = np.random.default_rng(seed)
        self.B, self.first, self.taken = B, first, 0
        self.lens = [int(rng.integers(0, hi + 1)) if r < live else 0 for r in range(B)]
        mb = width or -(-hi // 16) + 1
        own = sum(-(-n // 16) for n in self.lens)
        self.nb = first + own + spare
        self.free = list(range(first, self.nb))
        rng.shuffle(self.free)
        self.tables = [[-1] * mb for _ in range(B)]
        for r in range(live):
            for j in range(-(-self.lens[r] // 16)):
                if first and j < 2:
                    self.tables[r][j] = int(rng.integers(0, first))
                else:
                    self.tables[r][j] = self.free[self.taken]
                    self.taken += 1
        self.holds = [0] * (self.nb - first)
        words = -(-len(self.holds) // 32)
        self.d = dict(bt=dev(np.array(self.tables).reshape(B, mb)), lens=dev(self.lens), holds=dev(self.holds + [0] * words),
                      free=dev(self.free), taken=dev([self.taken]), src=dev([9] * B), dst=dev([9] * B), status=dev([9]),
                      out=dev([9]))

    def state(self, want_copies=None):
        torch.cuda.synchronize()
        d = self.d
        assert ints(d["bt"]) == self.tables and ints(d["lens"]) == self.lens
        assert ints(d["holds"]) == self.holds + [0] * -(-len(self.holds) // 32)
        assert ints(d["free"]) == self.free and ints(d["taken"]) == [self.taken]
        if want_copies:
            assert (ints(d["src"]), ints(d["dst"])) == want_copies

    def fork(self, sources, in_place=True):
        d = self.d
        out = d["taken"] if in_place else d["out"]
        ilpc.fork_tables(d["bt"], d["lens"], dev(sources), d["holds"], self.first, d["free"], d["taken"], d["src"],
                         d["dst"], out, d["status"], self.nb)
        *rest, self.taken_after, st = tree_ref.fork_ref(self.tables, self.lens, sources, self.holds, self.first,
                                                        self.free, self.taken, self.nb)
        self.tables, self.lens, self.holds, src, dst = rest
        torch.cuda.synchronize()
        assert ints(d["status"]) == [st] and ints(out) == [self.taken_after]
        self.taken = self.taken_after
        d["taken"] = out if in_place else out.clone()
        self.state((src, dst))
        return st

    def release(self, lens, in_place=True):
        d = self.d
        out = d["taken"] if in_place else d["out"]
        ilpc.release_shared(d["bt"], dev(lens), d["holds"], self.first, d["free"], d["taken"], out, d["status"], self.nb)
        self.holds, self.free, self.taken, st = tree_ref.release_shared_ref(self.tables, lens, self.holds, self.first,
                                                                            self.free, self.taken, self.nb)
        torch.cuda.synchronize()
        assert ints(d["status"]) == [st] and ints(out) == [self.taken]
        d["taken"] = out if in_place else out.clone()
        self.state()
        return st


@pytest.mark.parametrize("B,live,hi,first", [(2, 1, 40, 0), (4, 1, 16, 0), (16, 4, 350, 5), (64, 64, 100, 3), (300, 20, 90, 0),
                                             (1100, 100, 60, 7), (512, 64, 2000, 9), (7, 2, 30000, 0), (3000, 5, 33, 1)])
@pytest.mark.parametrize("in_place", [False, True])
def test_forks_and_releases(B, live, hi, first, in_place):
    rng = np.random.default_rng(B + hi)
    s = Rows(B, live, hi, first, B + 8, B)
    sources = [r if r < live or rng.random() < 0.1 else int(rng.integers(0, live)) for r in range(B)]
    assert s.fork(sources, in_place) == 0
    ended = [r for r in range(B) if rng.random() < 0.5]
    assert s.release([n if r in set(ended) else 0 for r, n in enumerate(s.lens)], in_place) == 0
    left = [0 if r in set(ended) else n for r, n in enumerate(s.lens)]
    assert s.release(left, in_place) == 0
    assert s.taken == 0 and sorted(s.free) == list(range(first, s.nb))


@pytest.mark.parametrize("B,live,spare", [(20, 6, 300000), (700, 30, 140000)])
def test_many_counted_blocks(B, live, spare):
    s = Rows(B, live, 400, 3, spare, B)
    sources = [r if r < live else r % live for r in range(B)]
    assert s.fork(sources) == 0
    assert s.release([n if r % 3 else 0 for r, n in enumerate(s.lens)]) == 0
    rest = [0 if r % 3 else n for r, n in enumerate(s.lens)]
    last = s.tables[0][-(-s.lens[0] // 16) - 1]
    s.tables[0] = list(s.tables[0])
    s.tables[0][2] = last  # once too often
    s.d["bt"].copy_(dev(s.tables))
    assert s.release(rest) == ilpc.NOT_HELD
    s.tables[0][2] = 1  # (not counted; what stood there stays held)
    s.d["bt"].copy_(dev(s.tables))
    assert s.release(rest) == 0 and s.taken <= 1


def test_forks_of_forks_and_of_lengths_at_block_ends():
    s = Rows(9, 1, 0, 2, 60, 0, width=8)
    for n, row in ((0, 0), (1, 0), (15, 0), (16, 0), (17, 0), (64, 0), (128, 0)):
        s.lens[0] = n
        s.tables[0] = [1] + [s.free[i] for i in range(s.taken, s.taken + 7)]
        s.tables[0] = s.tables[0][:-(-n // 16)] + [-1] * (8 - -(-n // 16))
        s.taken += max(-(-n // 16) - 1, 0)
        s.d["bt"].copy_(dev(s.tables)), s.d["lens"].copy_(dev(s.lens)), s.d["taken"].copy_(dev([s.taken]))
        assert s.fork([0, 0, 0, 3, 4, 5, 6, 7, 8]) == 0
        assert s.fork([0, 1, 2, 1, 2, 2, 0, 7, 8]) == 0
        assert s.release([x if r in (0, 2, 5) else 0 for r, x in enumerate(s.lens)]) == 0
        assert s.release([0 if r in (0, 2, 5) else x for r, x in enumerate(s.lens)]) == 0
        assert s.taken == 0
        s.lens = [0] * 9
        s.d["lens"].zero_()


@pytest.mark.parametrize("kind", ["blocks", "source", "low source", "source moves", "long", "negative", "taken",
                                  "taken low"])
@pytest.mark.parametrize("B", [12, 700])
def test_refused_forks_change_nothing(kind, B):
    s = Rows(B, 4, 100, 2, 40, 1)
    s.lens[:4] = [33, 20, 47, 5] if kind != "blocks" else [33] * 4
    need = max(-(-n // 16) for n in s.lens)
    s.tables = [row[:8] + [-1] * (8 - len(row)) for row in s.tables]
    s.d["bt"], s.d["lens"] = dev(s.tables), dev(s.lens)
    assert need <= 8
    src = list(range(B))
    src[5], src[B - 1] = 1, 2
    bit = ilpc.BAD_VALUE
    if kind == "blocks":
        src, bit = [0] + [0] * (B - 1), ilpc.NO_BLOCKS
        src[1:4] = [1, 2, 3]
        s.free = s.free[:s.taken + 3]
        s.d["free"] = dev(s.free)
    elif kind == "source":
        src[7] = B
    elif kind == "low source":
        src[7] = -1
    elif kind == "source moves":
        src[6] = 5
    elif kind == "long":
        s.lens[2], bit = 129, ilpc.TOO_LONG
    elif kind == "negative":
        s.lens[1] = -3
    elif kind == "taken":
        s.taken = len(s.free) + 1
    else:
        s.taken = -1
    s.d["lens"], s.d["taken"] = dev(s.lens), dev([s.taken])
    assert s.fork(src) & bit


@pytest.mark.parametrize("kind", ["twice", "too many", "long", "negative", "taken"])
@pytest.mark.parametrize("B", [12, 1500])
def test_refused_releases_change_nothing(kind, B):
    s = Rows(B, B // 2, 100, 2, B, 2)
    assert s.fork([r if r < B // 2 else r % (B // 2) for r in range(B)]) == 0
    lens, bit = list(s.lens), {"twice": ilpc.NOT_HELD, "too many": ilpc.NO_BLOCKS, "long": ilpc.TOO_LONG}.get(kind, 8)
    if kind == "twice":
        row = next(r for r in range(B // 2) if s.lens[r] > 48)
        s.tables[row] = list(s.tables[row])
        s.tables[row][-(-s.lens[row] // 16) - 1] = s.tables[row][2]
        s.d["bt"].copy_(dev(s.tables))
    elif kind == "too many":
        s.taken = 1
        s.d["taken"].fill_(1)
    elif kind == "long":
        lens[3] = 16 * len(s.tables[0]) + 1
    elif kind == "negative":
        lens[3] = -1
    else:
        s.taken = len(s.free) + 5
        s.d["taken"].fill_(s.taken)
    assert s.release(lens) & bit


def test_ids_outside_the_counted_blocks_are_shared_uncounted():
    s = Rows(3, 1, 0, 4, 20, 3, width=6)
    s.lens[0], s.tables[0] = 80, [1, 3, 4, 23, 1 << 30, -1]
    s.taken = 2
    s.nb = 24
    s.d["bt"].copy_(dev(s.tables)), s.d["lens"].copy_(dev(s.lens)), s.d["taken"].fill_(2)
    assert s.fork([0, 0, 0]) == 0 and s.holds[0] == 2 and s.holds[19] == 2
    assert s.release(s.lens) == 0 and s.taken == 0


def test_the_binding_refuses_overlaps_and_shapes():
    s = Rows(4, 2, 40, 2, 20, 4)
    d, src = s.d, dev([0, 1, 0, 1])
    fork = lambda **k: ilpc.fork_tables(**dict(dict(  # noqa: E731
        block_tables=d["bt"], seq_lens=d["lens"], sources=src, holds=d["holds"], first_id=2, free_ids=d["free"],
        taken=d["taken"], copy_src=d["src"], copy_dst=d["dst"], taken_out=d["out"], status=d["status"],
        num_blocks=s.nb), **k))
    for bad in (dict(copy_src=d["lens"]), dict(copy_dst=src), dict(status=d["taken"]), dict(taken_out=d["lens"][:1]),
                dict(holds=d["holds"][:-1]), dict(first_id=3), dict(first_id=-1), dict(num_blocks=s.nb + 1),
                dict(sources=src[:3]), dict(sources=src.long()), dict(first_id=s.nb + 1), dict(copy_src=d["free"][:4])):
        with pytest.raises(ilpc.ILPCError):
            fork(**bad)
    with pytest.raises(ilpc.ILPCError):
        ilpc.release_shared(d["bt"], d["lens"], d["holds"], 2, d["holds"][:3], d["taken"], d["out"], d["status"], s.nb)
    n = dev([-1, 0, 0, 1])
    cu, st = dev([0, 4]), dev([3])
    o = [dev([0] * 4)] + [dev([0]) for _ in range(4)]
    with pytest.raises(ilpc.ILPCError, match="overlap"):
        ilpc.tree_accept(n, n, n, cu, st, n, *o[1:])
    with pytest.raises(ilpc.ILPCError, match="overlap"):
        ilpc.tree_accept(n, n, n, cu, st, o[0], o[1], o[1], *o[3:])
    with pytest.raises(ilpc.ILPCError):
        ilpc.tree_accept(n, n[:3], n, cu, st, *o)
    with pytest.raises(ilpc.ILPCError):
        ilpc.tree_masks(n, cu, dev([[0]] * 3, np.int64))
    with pytest.raises(ilpc.ILPCError):
        ilpc.tree_masks(n, cu, dev([[0]] * 4, np.int64), n)
    with pytest.raises(ilpc.ILPCError):
        ilpc.tree_masks(n, cu, dev([[0] * 17] * 4, np.int64))
    s.state()


def test_no_request_at_all():
    e, one = dev([]), dev([0])
    bt, m = torch.zeros(0, 4, dtype=torch.int32, device="cuda"), torch.zeros(0, 1, dtype=torch.int64, device="cuda")
    kp, vp = pools(4, 2, 64)
    out, st, holds = dev([9]), dev([9]), dev([0, 0, 0])
    ilpc.tree_masks(e, one, m)
    ilpc.tree_accept(e, e, e, one, e, *[e.clone() for _ in range(5)])
    ilpc.kv_compact(kp, vp, bt, one, e, e, e)
    ilpc.copy_blocks(kp, vp, e, e)
    ilpc.fork_tables(bt, e, e.clone(), holds, 2, dev([2, 3]), dev([1]), e.clone(), e.clone(), out, st, 4)
    torch.cuda.synchronize()
    assert (ints(out), ints(st)) == ([1], [0])
    ilpc.release_shared(bt, e, holds, 2, dev([2, 3]), dev([1]), out, st, 4)
    torch.cuda.synchronize()
    assert (ints(out), ints(st)) == ([1], [0])
    # requests without nodes
    z, path = dev([0, 0]), [dev([9, 9]) for _ in range(4)]
    ilpc.tree_accept(e, e, e, dev([0, 0, 0]), dev([5, 16]), e.clone(), *path, root_targets=dev([7, 8]))
    torch.cuda.synchronize()
    assert [ints(p) for p in path] == [[0, 0], [7, 8], [5, 16], [1, 1]]
    del z


@pytest.mark.parametrize("n", [131072, 131073, 300001])
def test_no_row_to_release_over_many_blocks(n):
    bt, e = torch.zeros(0, 4, dtype=torch.int32, device="cuda"), dev([])
    holds = torch.zeros(ilpc.holds_words(n), dtype=torch.int32, device="cuda")
    holds[:n] = torch.arange(n, dtype=torch.int32, device="cuda") % 3
    want = holds.clone()
    free, out, st = dev([5, 6, 7]), dev([9]), dev([9])
    ilpc.release_shared(bt, e, holds, 2, free, dev([1]), out, st, n + 2)
    torch.cuda.synchronize()
    assert (ints(out), ints(st), ints(free)) == ([1], [0], [5, 6, 7]) and torch.equal(holds, want)
    ilpc.release_shared(bt, e, holds, 2, free, dev([4]), out, st, n + 2)
    torch.cuda.synchronize()
    assert (ints(out), ints(st)) == ([4], [ilpc.BAD_VALUE]) and torch.equal(holds, want)


# -- together: decoding by trees, and sampling several answers -----------------------

class Model:
    """A fixed next token, and K/V that depend on (token, position) alone."""

    def __init__(self, Hkv, D, vocab=40, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.next = np.random.default_rng(seed).permutation(vocab)
        rnd = lambda: torch.randn(vocab, Hkv, D, generator=g)  # noqa: E731
        self.k, self.v, self.vocab = rnd(), rnd(), vocab

    def kv(self, tokens, positions):
        t, p = np.asarray(tokens, int), torch.as_tensor(np.asarray(positions), dtype=torch.float32)[:, None, None]
        return ((self.k[t] * torch.cos(p * 0.1)).to(torch.bfloat16), (self.v[t] * torch.cos(p * 0.07)).to(torch.bfloat16))


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("shared", [False, True])
def test_speculative_decoding_leaves_the_cache_of_plain_decoding(captured, shared):
    Hq, Hkv, D, B, N = 8, 2, 64, 3, 21
    rng = np.random.default_rng(5)
    m = Model(Hkv, D)
    lens = [37, 5, 64]
    pc = pipeline.PagedPrefixCache(Hkv, D, 16, 20, B, 10, spare_blocks=40)
    prompts = [rng.integers(0, m.vocab, n).astype(np.int32) for n in lens]
    c, t = pc.match(prompts)
    b0 = pc.upload_prefill(c, t, lens)
    k, v = m.kv(np.concatenate(prompts), np.concatenate([np.arange(n) for n in lens]))
    pc.append(b0, k.cuda(), v.cuda())
    tab = pipeline.DeviceTables(pc, t, lens, B * N + 4, max_nodes=N, shared=shared)
    seqs = [list(p) for p in prompts]
    roots = [int(m.next[s[-1]]) for s in seqs]
    R = tab.max_rows
    d = dict(new=dev([0] * B), par=dev([0] * R), tok=dev([0] * R), pick=dev([0] * R))
    kv = [torch.zeros(R, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q, out = torch.randn(R, Hq, D, device="cuda").to(torch.bfloat16), torch.zeros(R, Hq, D, dtype=torch.bfloat16, device="cuda")

    def step():
        batch = tab.extend(d["new"], N)
        masks, _ = tab.tree(d["par"])
        pc.append_slots(tab.slot_map, *kv)
        pc.attend_tree(batch, q, out, D ** -0.5, masks)
        tab.accept(d["par"], d["tok"], d["pick"])
        pc.compact(batch, tab.path, tab.n_accepted)

    graph = None
    if captured:
        # (warmed up without new tokens, which changes nothing)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    for it in range(12):
        new, par, tok, pick, pos = [], [], [], [], []
        drafts = []
        for r in range(B):
            n = int(rng.integers(1, N + 1)) if it % 4 else (0 if r == 1 else 1)
            p = random_tree(n, rng, 2)
            tk = [0] * n
            for i in range(n):
                right = m.next[tk[p[i]]] if i else roots[r]
                tk[i] = int(right) if i == 0 or rng.random() < 0.6 else int(rng.integers(0, m.vocab))
            new.append(n)
            drafts.append((p, tk))
            par += p
            tok += tk
            pick += [int(m.next[x]) for x in tk]
            pos += [len(seqs[r]) + len(a) - 1 for a in tree_ref.ancestors(p)]
        n = len(par)
        d["new"].copy_(dev(new))
        for key, x in (("par", par), ("tok", tok), ("pick", pick)):
            d[key][:n] = dev(x)
        for dst, src in zip(kv, m.kv(tok, pos)):
            dst[:n] = src.cuda()
            dst[n:] = float("nan")
        if graph is None:
            step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        assert ints(tab.status) == [0]
        assert ints(tab.positions)[:n] == pos
        at = 0
        for r, (p, tk) in enumerate(drafts):
            path, nxt = tree_ref.accept_ref(p, tk, [int(m.next[x]) for x in tk])
            # attention of the nodes, over what plain decoding would have stored
            if p:
                keys = seqs[r]
                ck, cv = m.kv(keys + tk, list(range(len(keys))) + pos[at:at + len(p)])
                seen = np.zeros((len(p), len(p)), bool)
                for i, line in enumerate(tree_ref.ancestors(p)):
                    seen[i, line] = True
                ref, mag = tree_ref.tree_attention_ref(q[at:at + len(p)].float().cpu().numpy(), ck.float().numpy(),
                                                       cv.float().numpy(), D ** -0.5, seen)
                err = np.abs(out[at:at + len(p)].float().cpu().numpy() - ref)
                assert (err <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 * (1 + 2.0 ** -8) + 2.0 ** -13) * mag).all(), (it, r)
            seqs[r] += [tk[i] for i in path]
            if p:
                roots[r] = nxt
            assert ints(tab.next_tokens)[r] == nxt
            at += len(p)
        assert ints(tab.seq_lens) == [len(s) for s in seqs]
        # every block once: held by the rows, or free
        rows, taken = ints(tab.block_tables), ints(pc.free_taken)[0]
        used = [b for r in range(B) for b in rows[r][:-(-len(seqs[r]) // 16)]]
        assert len(set(used)) == len(used)
        assert sorted([b for b in used if b >= 16] + ints(pc.free_ids)[taken:]) == list(range(16, 56))
    # the cache holds the accepted sequences, as plain decoding would have stored them
    for r, s in enumerate(seqs):
        k, v = m.kv(s, np.arange(len(s)))
        row, at = rows[r], np.arange(len(s))
        blk = torch.tensor(row, device="cuda")[torch.tensor(at // 16, device="cuda")]
        off = torch.tensor(at % 16, device="cuda")
        assert same_bits(pc.k_pool[blk, :, off], k.cuda()) and same_bits(pc.v_pool[blk, :, :, off], v.cuda())
        assert s[-1] == (m.next[s[-2]] if len(s) > lens[r] + 1 else s[-1])
    tab.release(dev([1] * B))
    torch.cuda.synchronize()
    assert ints(pc.free_taken) == [0] and ints(tab.seq_lens) == [0] * B


@pytest.mark.parametrize("shared", [False, True])
def test_accept_gives_no_row_tokens_that_it_has_not(shared):
    pc = pipeline.PagedPrefixCache(1, 64, 4, 8, 3, 8, spare_blocks=30)
    tab = pipeline.DeviceTables(pc, np.full((3, 8), -1, np.int32), [0, 0, 0], 60, max_nodes=20, shared=shared)
    chain = list(range(-1, 19)) * 3
    par, tok, all_of, none = dev(chain), dev([3] * 60), dev([3] * 60), dev([4] * 60)
    tab.extend(dev([20, 20, 20]), 20)
    tab.release(dev([0, 1, 0]))
    # a request released before the draft is decided stays released
    tab.accept(par, tok, all_of)
    torch.cuda.synchronize()
    assert ints(tab.n_accepted) == [20] * 3 and ints(tab.seq_lens) == [20, 0, 20] and ints(pc.free_taken) == [4]
    # decided again: fewer, and then more than are left
    for picks in (none, all_of):
        tab.accept(par, tok, picks)
        torch.cuda.synchronize()
        assert ints(tab.status) == [0] and ints(tab.seq_lens) == [1, 0, 1] and ints(pc.free_taken) == [2]
    # an extend that is refused is no draft
    tab.extend(dev([20, 200, 20]), 200)
    tab.accept(par, tok, all_of)
    torch.cuda.synchronize()
    assert ints(tab.n_accepted) == [0] * 3 and ints(tab.seq_lens) == [1, 0, 1] and ints(pc.free_taken) == [2]
    rows, taken = ints(tab.block_tables), ints(pc.free_taken)[0]
    assert sorted([rows[0][0], rows[2][0]] + ints(pc.free_ids)[taken:]) == list(range(4, 34))


@pytest.mark.parametrize("lens", [[37, 5], [64, 16], [30, 0]])
def test_sampling_several_answers_of_each_prompt(lens):
    Hq, Hkv, D, B = 8, 2, 64, 8
    rng = np.random.default_rng(6)
    m = Model(Hkv, D)
    pc = pipeline.PagedPrefixCache(Hkv, D, 16, 20, B, 10, spare_blocks=60)
    prompts = [rng.integers(0, m.vocab, n).astype(np.int32) for n in lens]
    live = [p for p in prompts if len(p)]
    c, t = pc.match(live)
    k, v = m.kv(np.concatenate(live), np.concatenate([np.arange(len(p)) for p in live]))
    pc.append(pc.upload_prefill(c, t, [len(p) for p in live]), k.cuda(), v.cuda())
    tables = np.full((B, 20), -1, np.int32)
    tables[:len(live)] = t
    tab = pipeline.DeviceTables(pc, tables, [len(p) for p in live] + [0] * (B - len(live)), B, shared=True)
    src, dst = tab.fork(dev([0, 1, 0, 0, 1, 1, 0, 7]))
    pc.copy_blocks(src, dst)
    of = [0, 1, 0, 0, 1, 1, 0]
    seqs = [list(prompts[p]) for p in of] + [[]]
    q, out = torch.randn(B, Hq, D, device="cuda").to(torch.bfloat16), torch.zeros(B, Hq, D, dtype=torch.bfloat16, device="cuda")
    alive = [True] * 7 + [False]
    for it in range(40):
        tok = rng.integers(0, m.vocab, B).tolist()
        new = [int(a) for a in alive]
        batch = tab.extend(dev(new), 1)
        rows = [r for r in range(B) if alive[r]]
        k, v = m.kv([tok[r] for r in rows], [len(seqs[r]) for r in rows])
        pad = torch.full((B - len(rows), Hkv, D), float("nan"), dtype=torch.bfloat16)
        tab.append(torch.cat([k, pad]).cuda(), torch.cat([v, pad]).cuda())
        pc.attend(batch, q, out, D ** -0.5)
        for r in rows:
            seqs[r].append(tok[r])
        torch.cuda.synchronize()
        assert ints(tab.status) == [0]
        if it in (5, 20):  # two answers end; at 20 their rows become forks of a living one
            end = [r for r in (1, 3) if alive[r]] if it == 5 else [r for r in (0, 6) if alive[r]]
            tab.release(dev([int(r in end) for r in range(B)]))
            for r in end:
                alive[r], seqs[r] = False, []
        if it == 25:
            s, d = tab.fork(dev([2 if r in (0, 3) else r for r in range(B)]))
            pc.copy_blocks(s, d)
            for r in (0, 3):
                alive[r], seqs[r] = True, list(seqs[2])
        torch.cuda.synchronize()
        assert ints(tab.seq_lens) == [len(s) for s in seqs]
    tables = ints(tab.block_tables)
    count = {}
    for r in range(B):
        s = seqs[r]
        if not s:
            continue
        k, v = m.kv(s, np.arange(len(s)))
        at = np.arange(len(s))
        blk = torch.tensor(tables[r], device="cuda")[torch.tensor(at // 16, device="cuda")]
        off = torch.tensor(at % 16, device="cuda")
        assert same_bits(pc.k_pool[blk, :, off], k.cuda()) and same_bits(pc.v_pool[blk, :, :, off], v.cuda())
        for b in tables[r][:-(-len(s) // 16)]:
            count[b] = count.get(b, 0) + 1
    holds, taken = ints(pc.holds), ints(pc.free_taken)[0]
    assert all(holds[b - 16] == max(count.get(b, 0) - 1, 0) for b in range(16, 76)) and not any(holds[60:])
    assert sorted([b for b in count if b >= 16] + ints(pc.free_ids)[taken:]) == list(range(16, 76))
    tab.release(dev([1] * B))
    torch.cuda.synchronize()
    assert ints(pc.free_taken) == [0] and not any(ints(pc.holds))


def test_device_tables_say_what_they_were_made_without():
    pc = pipeline.PagedPrefixCache(1, 64, 4, 4, 2, 6, spare_blocks=4)
    tab = pipeline.DeviceTables(pc, np.full((2, 4), -1, np.int32), [0, 0], 2)
    z = dev([0, 0])
    for call in (lambda: tab.tree(z), lambda: tab.accept(z, z, z), lambda: tab.fork(z)):
        with pytest.raises(ilpc.ILPCError, match="was made without"):
            call()
    assert release_ref([[1]], [0], [0], [], 0)[-1] == 0


@pytest.mark.parametrize("case", ["plan", "forks"])
def test_captured_calls_follow_their_inputs(case):
    if case == "plan":
        rng = np.random.default_rng(0)
        par, tok = dev([-1] * 20), dev(range(20))
        cu, start, masks, pos = dev([0, 12, 20]), dev([3, 40]), dev(np.zeros((20, 1)), np.int64), dev([0] * 20)
        pick, outs = dev([0] * 20), [dev([0] * 20)] + [dev([0, 0]) for _ in range(4)]

        def calls():
            ilpc.tree_masks(par, cu, masks, pos, start)
            ilpc.tree_accept(par, tok, pick, cu, start, *outs)
            return [masks, pos] + outs
    else:
        s = Rows(40, 5, 300, 2, 300, 5)
        d = s.d
        src, ended = dev(range(40)), dev([0] * 40)

        def calls():
            ilpc.fork_tables(d["bt"], d["lens"], src, d["holds"], 2, d["free"], d["taken"], d["src"], d["dst"], d["taken"],
                             d["status"], s.nb)
            ilpc.release_shared(d["bt"], ended, d["holds"], 2, d["free"], d["taken"], d["taken"], d["status"], s.nb)
            return list(d.values())
    calls()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for k in range(4):
        if case == "plan":
            p = random_tree(12, rng, 2) + random_tree(8, rng, 1)
            par.copy_(dev(p))
            pick.copy_(dev(picks_for(p, list(range(20)), rng)))
        else:
            src.copy_(dev([r if r < 5 or r % 7 == k else r % 5 for r in range(40)]))
            ended.copy_(dev([0 if r < 5 or r % 7 == k else int(d["lens"][r % 5]) for r in range(40)]))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in calls()]
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, calls()))


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("rooted", [False, True])
def test_accept_leaves_a_refused_extend_to_be_read(captured, shared, rooted):
    # one read a step has to tell a refused extend from a draft of which nothing was accepted
    pc = pipeline.PagedPrefixCache(1, 64, 4, 8, 2, 8, spare_blocks=12)
    tab = pipeline.DeviceTables(pc, np.full((2, 8), -1, np.int32), [0, 0], 60, max_nodes=20, shared=shared)
    new, par, tok, pick = dev([0, 0]), dev(list(range(-1, 29)) * 2), dev([3] * 60), dev([3] * 60)
    root = dev([3, 3]) if rooted else None

    def step():
        tab.extend(new, 20)
        tab.accept(par, tok, pick, root)

    step()
    torch.cuda.synchronize()
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    # refused: a request past its table, more rows than there are, no block left
    for lens, bit, after in (([9, 12], 0, [9, 12]),
                             ([200, 1], ilpc.NO_BLOCKS | ilpc.TOO_LONG | ilpc.TOO_MANY_ROWS, [9, 12]),
                             ([1, 9], 0, [10, 21]), ([31, 30], ilpc.TOO_MANY_ROWS, [10, 21]), ([0, 0], 0, [10, 21]),
                             ([-1, 3], ilpc.BAD_VALUE, [10, 21]), ([4, 0], 0, [14, 21])):
        new.copy_(dev(lens))
        p = sum((list(range(-1, max(n, 0) - 1)) for n in lens), [])[:60]
        par[:len(p)] = dev(p)
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        assert ints(tab.status) == [bit] and ints(tab.seq_lens) == after, lens
        if bit:
            assert ints(tab.n_accepted) == [0, 0]
    pc.free_ids = pc.free_ids[:3]
    if not captured:
        new.copy_(dev([20, 20]))
        step()
        torch.cuda.synchronize()
        assert ints(tab.status) == [ilpc.NO_BLOCKS] and ints(tab.seq_lens) == [14, 21]


def test_what_accept_itself_refuses_is_added():
    pc = pipeline.PagedPrefixCache(1, 64, 4, 8, 1, 8, spare_blocks=12)
    tab = pipeline.DeviceTables(pc, np.full((1, 8), -1, np.int32), [0], 60, max_nodes=20)
    tab.extend(dev([20]), 20)
    pc.free_taken.fill_(0)  # (not by any call of the class)
    par, tok, none = dev(list(range(-1, 59))), dev([3] * 60), dev([4] * 60)
    tab.accept(par, tok, none)
    torch.cuda.synchronize()
    assert ints(tab.status) == [ilpc.NO_BLOCKS] and ints(tab.seq_lens) == [20] and ints(pc.free_taken) == [0]
    pc.free_taken.fill_(2)
    tab.extend(dev([0]), 20)
    torch.cuda.synchronize()
    assert ints(tab.status) == [0] and ints(tab.seq_lens) == [20]


# -- forks beside drafts ---------------------------------------------------------------

def conserved(pc, tab):
    """Every spare block is free or held by as many rows as its count says."""
    torch.cuda.synchronize()
    rows, lens, held = ints(tab.block_tables), ints(tab.seq_lens), {}
    for row, n in zip(rows, lens):
        for b in row[:-(-n // 16)]:
            held[b] = held.get(b, 0) + 1
    nb, first, taken = pc.k_pool.shape[0], pc.num_blocks, ints(pc.free_taken)[0]
    assert sorted([b for b in held if b >= first] + ints(pc.free_ids)[taken:]) == list(range(first, nb))
    assert ints(pc.holds)[:nb - first] == [max(held.get(b, 0) - 1, 0) for b in range(first, nb)]


def rows_of_cache(pc, tab, r):
    at = torch.arange(ints(tab.seq_lens)[r], device="cuda")
    blk, off = tab.block_tables[r].long()[at // 16], at % 16
    return pc.k_pool[blk, :, off].clone(), pc.v_pool[blk, :, :, off].clone()


def drafting(lens, B=5, N=24):
    """A table of B rows that hold `lens` tokens, over a cache of random bits."""
    pc = pipeline.PagedPrefixCache(2, 64, 4, 12, B, 12, spare_blocks=50)
    for pool, x in zip((pc.k_pool, pc.v_pool), pools(54, 2, 64)):
        pool.copy_(x)
    tab = pipeline.DeviceTables(pc, np.full((B, 12), -1, np.int32), [0] * B, B * 40, max_nodes=N, shared=True)
    tab.extend(dev(lens), 64)
    return pc, tab, dict(par=dev(list(range(-1, 39)) * B), tok=dev([3] * 40 * B), yes=dev([3] * 40 * B), no=dev([4] * 40 * B))


@pytest.mark.parametrize("picks", ["yes", "no"])
@pytest.mark.parametrize("rooted", [False, True])
def test_a_fork_ends_the_open_drafts_of_its_rows(picks, rooted):
    # rows 0 and 1 are forked from while their drafts are open: their blocks are the forks' as well
    pc, tab, d = drafting([37, 16, 20, 0, 0])
    new = [24, 24, 21, 0, 0]
    batch = tab.extend(dev(new), 24)
    par = dev(sum((list(range(-1, n - 1)) for n in new), []) + [0] * (tab.max_rows - sum(new)))
    if picks == "yes":  # a path that leaves nodes out: its rows would move
        par[2:24], par[26:48], par[50:69] = 0, 0, 0
        pick, tok = dev([7] * tab.max_rows), dev([3] * tab.max_rows)
        for a, n in zip((0, 24, 48), new):
            tok[a + n - 1] = 7
    else:
        pick, tok = d["no"], d["tok"]
    pc.copy_blocks(*tab.fork(dev([0, 1, 2, 0, 1])))
    torch.cuda.synchronize()
    assert ints(tab.status) == [0]
    conserved(pc, tab)
    before = [rows_of_cache(pc, tab, r) for r in (0, 1, 3, 4)]
    tab.accept(par, tok, pick, dev([3] * 5) if rooted else None)
    pc.compact(batch, tab.path, tab.n_accepted)
    torch.cuda.synchronize()
    n2 = {"yes": 2, "no": 1}[picks]
    assert ints(tab.status) == [0] and ints(tab.seq_lens) == [61, 40, 20 + n2, 61, 40]
    assert ints(tab.n_accepted) == [0, 0, n2, 0, 0] and ints(tab.path)[:48] == [-1] * 48
    assert ints(tab.next_tokens)[3:] == [3 if rooted else -1] * 2
    conserved(pc, tab)
    for r, (k, v) in zip((0, 1, 3, 4), before):
        assert all(same_bits(a, b) for a, b in zip(rows_of_cache(pc, tab, r), (k, v))), r
    # the next draft of these rows is a draft again
    tab.extend(dev([20, 20, 0, 20, 0]), 20)
    chain = dev(list(range(-1, 19)) * 3 + [0] * (tab.max_rows - 60))
    tab.accept(chain, d["tok"], d["no"])
    torch.cuda.synchronize()
    assert ints(tab.status) == [0] and ints(tab.seq_lens) == [62, 41, 20 + n2, 62, 40]
    conserved(pc, tab)


@pytest.mark.parametrize("picks", ["yes", "no"])
def test_a_row_forked_over_while_its_draft_is_open_keeps_its_sources_tokens(picks):
    for lens in ([20, 60, 5, 0, 0], [20, 64, 5, 0, 0], [50, 49, 5, 0, 0]):
        pc, tab, d = drafting(lens)
        batch = tab.extend(dev([18, 0, 18, 0, 0]), 18)
        tab.release(dev([1, 0, 0, 0, 0]))
        pc.copy_blocks(*tab.fork(dev([1, 1, 2, 3, 4])))
        torch.cuda.synchronize()
        before = [rows_of_cache(pc, tab, r) for r in (0, 1)]
        assert all(same_bits(a, b) for a, b in zip(*before))
        chain = dev(list(range(-1, 17)) * 2 + [0] * (tab.max_rows - 36))
        tab.accept(chain, d["tok"], d[picks])
        pc.compact(batch, tab.path, tab.n_accepted)
        torch.cuda.synchronize()
        k = 18 if picks == "yes" else 1
        assert ints(tab.status) == [0] and ints(tab.seq_lens) == [lens[1], lens[1], 5 + k, 0, 0]
        conserved(pc, tab)
        for r in (0, 1):
            assert all(same_bits(a, b) for a, b in zip(rows_of_cache(pc, tab, r), before[r])), r
        tab.release(dev([1] * 5))
        torch.cuda.synchronize()
        assert ints(pc.free_taken) == [0] and not any(ints(pc.holds))


def test_a_path_of_before_moves_nothing_in_a_row_forked_over():
    pc, tab, d = drafting([20, 52, 5, 0, 0])
    batch = tab.extend(dev([24, 0, 0, 0, 0]), 24)
    par = dev([-1, 0] + [0] * 21 + [0] + [0] * (tab.max_rows - 24))
    tok, pick = dev([3] * tab.max_rows), dev([9] * tab.max_rows)
    tok[23] = 9  # nodes 0 and 23 stay
    tab.accept(par, tok, pick)
    tab.release(dev([1, 0, 0, 0, 0]))
    pc.copy_blocks(*tab.fork(dev([1, 1, 2, 3, 4])))
    torch.cuda.synchronize()
    before = [rows_of_cache(pc, tab, r) for r in (0, 1)]
    pc.compact(batch, tab.path, tab.n_accepted)
    torch.cuda.synchronize()
    conserved(pc, tab)
    for r in (0, 1):
        assert all(same_bits(a, b) for a, b in zip(rows_of_cache(pc, tab, r), before[r])), r


def test_a_refused_fork_ends_no_draft():
    pc, tab, d = drafting([20, 33, 5, 0, 0])
    tab.extend(dev([20, 20, 20, 0, 0]), 20)
    for bad in ([0, 1, 2, 7, 4], [0, 1, 2, -1, 0], [0, 0, 2, 1, 4]):
        tab.fork(dev(bad))
        torch.cuda.synchronize()
        assert ints(tab.status) == [ilpc.BAD_VALUE] and ints(tab.start_pos) == [20, 33, 5, 0, 0]
    tab.fork(dev([0, 1, 2, 3, 4]))
    tab.accept(dev(list(range(-1, 19)) * 3 + [0] * (tab.max_rows - 60)), d["tok"], d["no"])
    torch.cuda.synchronize()
    assert ints(tab.status) == [0] and ints(tab.seq_lens) == [21, 34, 6, 0, 0] and ints(tab.n_accepted) == [1, 1, 1, 0, 0]
    conserved(pc, tab)


def test_requests_without_a_draft_keep_all():
    par, tok = [-1, 0, 1, -1, 0], [3] * 5
    for root, nxt in ((None, [3, -1, -1]), ([3, 8, 9], [3, 8, 9])):
        got = run_accept(par + [0], tok + [0], tok + [0], [0, 3, 5, 5], [7, -1, -1 << 31], root)
        most = (1 << 31) - 1
        assert got == [[0, 1, 2, -1, -1, 9], [3, 0, 0], nxt, [10, most, most], [1, most, most]]


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("lens", [[37, 5, 64], [16, 48, 0]])
def test_drafts_compacted_then_forked_then_drafted_again(lens, captured):
    # accept, compact, (release,) fork, copy_blocks, extend: each row's cache stays that of its accepted tokens
    Hkv, D, B, N = 2, 64, 6, 20
    rng = np.random.default_rng(sum(lens))
    m = Model(Hkv, D)
    pc = pipeline.PagedPrefixCache(Hkv, D, 16, 24, B, 10, spare_blocks=100)
    live = [rng.integers(0, m.vocab, n).astype(np.int32) for n in lens if n]
    c, t = pc.match(live)
    k, v = m.kv(np.concatenate(live), np.concatenate([np.arange(len(p)) for p in live]))
    pc.append(pc.upload_prefill(c, t, [len(p) for p in live]), k.cuda(), v.cuda())
    tables = np.full((B, 24), -1, np.int32)
    tables[:len(live)] = t
    tab = pipeline.DeviceTables(pc, tables, [len(p) for p in live] + [0] * (B - len(live)), B * N, max_nodes=N, shared=True)
    seqs = [list(p) for p in live] + [[]] * (B - len(live))
    R = tab.max_rows
    d = {k: dev([0] * R) for k in ("par", "tok", "pick")}
    new, ended, src = dev([0] * B), dev([0] * B), dev(range(B))
    kv = [torch.zeros(R, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def draft():
        batch = tab.extend(new, N)
        pc.append_slots(tab.slot_map, *kv)
        tab.accept(d["par"], d["tok"], d["pick"])
        pc.compact(batch, tab.path, tab.n_accepted)

    def fork():
        tab.release(ended)
        pc.copy_blocks(*tab.fork(src))

    calls = dict(draft=draft, fork=fork)
    if captured:
        for name, call in list(calls.items()):
            call()  # (without new tokens, ended rows or forks, which changes nothing)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                call()
            calls[name] = g.replay
    for it in range(14):
        sizes, par, tok, pick, pos = [], [], [], [], []
        for r in range(B):
            n = int(rng.integers(0, N + 1)) if seqs[r] else 0
            p = random_tree(n, rng, 2)
            tk = rng.integers(0, m.vocab, n).tolist()
            sizes.append(n)
            par, tok, pick = par + p, tok + tk, pick + picks_for(p, tk, rng, vocab=m.vocab)
            pos += [len(seqs[r]) + len(a) - 1 for a in tree_ref.ancestors(p)]
        n = len(par)
        new.copy_(dev(sizes))
        for key, x in (("par", par), ("tok", tok), ("pick", pick)):
            d[key][:n] = dev(x)
        for to, x in zip(kv, m.kv(tok, pos)):
            to[:n], to[n:] = x.cuda(), float("nan")
        calls["draft"]()
        torch.cuda.synchronize()
        assert ints(tab.status) == [0]
        at = 0
        for r in range(B):
            path, _ = tree_ref.accept_ref(*(x[at:at + sizes[r]] for x in (par, tok, pick)))
            seqs[r] = seqs[r] + [tok[at + i] for i in path]
            at += sizes[r]
        if it % 3 != 2:
            ends = [r for r in range(B) if seqs[r] and rng.random() < 0.35][:B - 2]
            for r in ends:
                seqs[r] = []
            on = [r for r in range(B) if seqs[r]]
            of = [r if seqs[r] or not on or rng.random() < 0.3 else int(rng.choice(on)) for r in range(B)]
            ended.copy_(dev([int(r in ends) for r in range(B)])), src.copy_(dev(of))
            calls["fork"]()
            torch.cuda.synchronize()
            assert ints(tab.status) == [0]
            seqs = [list(seqs[s]) for s in of]
        assert ints(tab.seq_lens) == [len(s) for s in seqs]
        for r, s in enumerate(seqs):
            if s:
                k, v = m.kv(s, np.arange(len(s)))
                got = rows_of_cache(pc, tab, r)
                assert same_bits(got[0], k.cuda()) and same_bits(got[1], v.cuda()), (it, r)
        conserved(pc, tab)
        if not any(seqs):
            break
    assert it > 3
    tab.release(dev([1] * B))
    torch.cuda.synchronize()
    assert ints(pc.free_taken) == [0] and not any(ints(pc.holds))


# -- replays ---------------------------------------------------------------------------

@pytest.mark.parametrize("words", [1, 3])
def test_replays_alone_write_masks_and_paths(words):
    # (outputs are spoiled before each replay, and read before anything else runs)
    rng = np.random.default_rng(words)
    sizes, n = ([12, 8], 20) if words == 1 else ([150, 40], 190)
    par, tok, pick, start = dev([-1] * n), dev(range(n)), dev([0] * n), dev([3, 40])
    cu, masks, pos = dev([0, sizes[0], n]), dev(np.zeros((n, words)), np.int64), dev([0] * n)
    outs = [dev([0] * n)] + [dev([0, 0]) for _ in range(4)]

    def calls():
        ilpc.tree_masks(par, cu, masks, pos, start)
        ilpc.tree_accept(par, tok, pick, cu, start, *outs)

    calls()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for k in range(5):
        trees = [random_tree(s, rng, 1 + k % 3) for s in sizes]
        p, s = sum(trees, []), rng.integers(0, 900, 2).tolist()
        t = picks_for(p[:sizes[0]], list(range(sizes[0])), rng) + picks_for(p[sizes[0]:], list(range(sizes[0], n)), rng)
        for x, y in ((par, p), (pick, t), (start, s)):
            x.copy_(dev(y))
        for x in [masks, pos] + outs:
            x.fill_(-77)
        g.replay()
        torch.cuda.synchronize()
        want_m, want_p, path, rest = [], [], [], [[], [], [], []]
        for at, tree, st in zip((0, sizes[0]), trees, s):
            m, q = tree_ref.masks_ref(tree, st, words)
            want_m += [signed(x) for x in m]
            want_p += q
            got, nxt = tree_ref.accept_ref(tree, list(range(at, at + len(tree))), t[at:at + len(tree)])
            path += got + [-1] * (len(tree) - len(got))
            for o, x in zip(rest, (len(got), nxt, st + len(got), -(-(st + len(got)) // 16))):
                o.append(x)
        assert ints(masks) == want_m and ints(pos) == want_p and [ints(o) for o in outs] == [path] + rest
        torch.zeros(1000, device="cuda").sum().item()  # (eager work between replays)


@pytest.mark.parametrize("B,live,hi", [(40, 5, 300), (400, 30, 500)])
def test_replays_alone_fork_copy_and_release(B, live, hi):
    # of one launch each and of two
    rng = np.random.default_rng(B)
    s = Rows(B, live, hi, 2, B + 200, 5)
    kp, vp = pools(s.nb, 2, 64)
    src, ended, d = dev(range(B)), dev([0] * B), s.d

    def calls():
        ilpc.fork_tables(d["bt"], d["lens"], src, d["holds"], 2, d["free"], d["taken"], d["src"], d["dst"], d["taken"],
                         d["status"], s.nb)
        ilpc.copy_blocks(kp, vp, d["src"], d["dst"])
        ilpc.release_shared(d["bt"], ended, d["holds"], 2, d["free"], d["taken"], d["taken"], d["out"], s.nb)

    calls()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    free_rows = set(range(live, B))
    for k in range(5):
        # some empty rows become forks, and some rows that hold something end
        sources = [int(rng.integers(0, live)) if r in free_rows and rng.random() < 0.5 else r for r in range(B)]
        *rest, taken, st = tree_ref.fork_ref(s.tables, s.lens, sources, s.holds, 2, s.free, s.taken, s.nb)
        s.tables, s.lens, s.holds, cs, cd = rest
        ends = [n if r >= live and rng.random() < 0.6 else 0 for r, n in enumerate(s.lens)]
        s.holds, s.free, s.taken, st2 = tree_ref.release_shared_ref(s.tables, ends, s.holds, 2, s.free, taken, s.nb)
        assert (st, st2) == (0, 0)
        src.copy_(dev(sources)), ended.copy_(dev(ends))
        for x in ("src", "dst", "status", "out"):
            d[x].fill_(-77)
        wk, wv = kp.clone(), vp.clone()
        for a, b in zip(cs, cd):
            if a >= 0 and b >= 0:
                wk[b], wv[b] = kp[a], vp[a]
        g.replay()
        torch.cuda.synchronize()
        assert ints(d["status"]) == [0] and ints(d["out"]) == [0]
        s.state((cs, cd))
        assert same_bits(kp, wk) and same_bits(vp, wv)
        # the rows that ended hold nothing from here on
        s.lens = [0 if e else n for e, n in zip(ends, s.lens)]
        d["lens"].copy_(dev(s.lens))
        free_rows = {r for r in range(live, B) if s.lens[r] == 0}
    assert any(s.holds)


# -- drafts' starts in the fork's own call ---------------------------------------------

@pytest.mark.parametrize("general", [False, True])
@pytest.mark.parametrize("B,live,hi", [(1, 1, 20), (12, 4, 100), (300, 40, 700), (3000, 5, 33)])
def test_forks_write_down_whose_drafts_have_ended(B, live, hi, general):
    rng = np.random.default_rng(B)
    for share in (0.0, 0.5, 1.0):
        s = Rows(B, live, hi, 2, B + 8, B)
        src = [int(rng.integers(0, live)) if r >= live and rng.random() < share else r for r in range(B)]
        d, start = s.d, rng.integers(0, 99, B).tolist()
        at = dev(start + [5])[:B]
        num = np.int64(s.nb) if general else s.nb  # (what is no plain int goes by way of ctypes)
        fork = lambda to, of=None: ilpc.fork_tables(  # noqa: E731
            d["bt"], d["lens"], dev(of or src), d["holds"], 2, d["free"], d["taken"], d["src"], d["dst"], d["taken"],
            d["status"], num, start_pos=to)
        if B > 1:
            fork(at, src[:-1] + [B])
            torch.cuda.synchronize()
            assert ints(d["status"]) == [ilpc.BAD_VALUE] and ints(at) == start
        fork(at)
        s.tables, s.lens, s.holds, cs, cd, s.taken, st = tree_ref.fork_ref(s.tables, s.lens, src, s.holds, 2, s.free, s.taken,
                                                                          s.nb)
        s.state((cs, cd))
        touched = {r for r in range(B) if src[r] != r} | {x for r, x in enumerate(src) if x != r}
        assert st == 0 and ints(d["status"]) == [0] and ints(at) == [-1 if r in touched else x for r, x in enumerate(start)]
        for bad in (at.long(), dev(start + [1]), d["lens"], d["src"]):
            with pytest.raises(ilpc.ILPCError):
                fork(bad)
        s.state((cs, cd))
