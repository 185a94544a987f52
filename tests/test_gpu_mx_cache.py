"""The paged cache in 4 bits against the oracle (float64): stores and reads byte by byte, the decode step to its rounding.

Tolerance of a decode output o = sum_j w_j v_j, with W = sum_j w_j |v_j|: its own rounding to bfloat16, half a step, 2^-8 |o|; the
probabilities' rounding to bfloat16, 2^-8 W at most (2^-9 of each would be the mean); scores are float32 sums of Dh exact products, off by Dh 2^-23 of
A = scale * sum |q| |k| at most, and the exponential's argument and result by a few more 2^-23 of the argument's magnitude (at most 2 A), which
moves weights, and their sum, by twice that: 2 (Dh + 16) 2^-23 A W; float32 sums over n tokens, n 2^-23 W at most each for numerator and
denominator: 2 n 2^-23 W."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2412_00876_amd as P
from oracle import mx_ref as R

DEV = "cuda:0"


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    return t if dtype is None else t.to(dtype)


def f64(t):
    return t.double().cpu().numpy()


def i32(a):
    return dev(np.asarray(a, np.int32))


CODE = {torch.float32: P.F32, torch.bfloat16: P.BF16}


class Path:
    """A cache on the device and its twin in the oracle; slots that hold no token are filled with `junk`."""

    def __init__(self, rs, B, mp, H, Dh, junk=0xFF, spare=3):
        self.B, self.H, self.Dh, self.cap = B, H, Dh, 16 * mp
        table = rs.permutation(B * mp + spare)[:B * mp].reshape(B, mp).astype(np.int32)
        pages = np.full((B * mp + spare, H, 17 * Dh), junk, np.uint8)
        self.pages, self.len = dev(pages), torch.zeros(B, dtype=torch.int32, device=DEV)
        self.cache = P.KVCache(self.pages, dev(table), self.len)
        self.ref = R.Cache(pages, table, np.zeros(B))
        self.err = torch.zeros(1, dtype=torch.int32, device=DEV)

    def fill(self, rs, lens):
        """Tokens of the given lengths, through the oracle."""
        for b, n in enumerate(lens):
            k, v = rs.standard_normal((2, n, self.H, self.Dh)).astype(np.float32)
            for t in range(n):
                self.ref.put(b, t, k[t], v[t])
        self.ref.lens = np.asarray(lens, np.int64)
        self.pages.copy_(dev(self.ref.pages))
        self.len.copy_(i32(lens))

    def same(self):
        assert np.array_equal(self.pages.cpu().numpy(), self.ref.pages)
        assert np.array_equal(self.len.cpu().numpy(), self.ref.lens)


# ---- store and load ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,Dh", [(1, 64), (3, 128), (5, 64), (8, 128)])
@pytest.mark.parametrize("gather", [False, True])
def test_store_and_load(H, Dh, dtype, gather):
    rs = np.random.default_rng(H * Dh + gather)
    lens, start = [5, 0, 16, 1, 33, 40, 17], [0, 7, 0, 15, 31, 3, 16]
    B, rows = len(lens), sum(lens)
    s = Path(rs, B, 5, H, Dh)
    off = np.cumsum([0] + lens)
    src_off = np.cumsum([0] + [2 * n + 1 for n in lens])
    src_idx = np.concatenate([np.sort(rs.permutation(2 * n + 1)[:n]) for n in lens]).astype(np.int32)
    total = src_off[-1] if gather else rows
    ld = H * Dh + 8
    kv = [torch.full((total, ld), float("nan"), dtype=dtype, device=DEV) for _ in range(2)]
    for t in kv:
        t[:, :H * Dh] = dev(rs.standard_normal((total, H * Dh)))
    P.dllava_mx_cache_store(kv[0], kv[1], ld, B, i32(off), i32(start), rows, i32(src_off) if gather else None, i32(src_idx) if gather else None,
                            s.cache, s.err, CODE[dtype])
    K, V = (f64(t[:, :H * Dh]).reshape(-1, H, Dh) for t in kv)
    for b in range(B):
        for i in range(lens[b]):
            at = src_off[b] + src_idx[off[b] + i] if gather else off[b] + i
            s.ref.put(b, start[b] + i, K[at], V[at])
        s.ref.lens[b] = start[b] + lens[b]
    s.same()                                                # nothing else was written
    assert int(s.err) == 0
    # back: three positions more than were stored, which are zeros, in both types
    n2 = [n + 3 for n in lens]
    off2 = np.cumsum([0] + n2)
    for out in (torch.bfloat16, torch.float32):
        ko, vo = (torch.full((off2[-1] + 2, ld), 9.0, dtype=out, device=DEV) for _ in range(2))
        P.dllava_mx_cache_load(s.cache, B, i32(off2), i32(start), int(off2[-1]), ko, vo, ld, CODE[out])
        for b in range(B):
            for i in range(n2[b]):
                want = s.ref.get(b, start[b] + i) if i < lens[b] else (0.0, 0.0)
                for t, w in zip((ko, vo), want):
                    assert np.array_equal(f64(t[off2[b] + i, :H * Dh]).reshape(H, Dh), np.broadcast_to(w, (H, Dh)))
        assert (ko[:, H * Dh:] == 9.0).all() and (ko[off2[-1]:] == 9.0).all() and (vo[off2[-1]:] == 9.0).all()


def test_store_beyond_the_capacity():
    rs = np.random.default_rng(1)
    s = Path(rs, 2, 2, 2, 64, junk=0)
    k = dev(rs.standard_normal((60, 2, 64))).bfloat16()
    P.dllava_mx_cache_store(k, k, 128, 2, i32([0, 40, 60]), i32([0, 20]), 60, None, None, s.cache, s.err, P.BF16)
    for b, (n, st, r0) in enumerate(((40, 0, 0), (20, 20, 40))):
        for i in range(n):
            if st + i < 32:
                s.ref.put(b, st + i, f64(k[r0 + i]), f64(k[r0 + i]))
        s.ref.lens[b] = 32
    s.same()
    assert int(s.err) == 1
    out = torch.full((60, 2, 64), 3.0, dtype=torch.bfloat16, device=DEV)   # positions behind the capacity read as zeros
    P.dllava_mx_cache_load(s.cache, 2, i32([0, 40, 60]), i32([0, 20]), 60, out, out.clone(), 128, P.BF16)
    empty = (out == 0).all(-1).all(-1)
    assert torch.nonzero(empty)[:, 0].tolist() == [*range(32, 40), *range(52, 60)]


@pytest.mark.parametrize("B", [64, 65, 130, 4200])
def test_store_and_load_of_many_sequences(B):
    """More sequences than are looked through at once, most of them short, some empty, also the first and the last."""
    rs = np.random.default_rng(B)
    lens, start = rs.integers(0, 4, B), rs.integers(0, 15, B)
    lens[[0, 1, B - 1]] = 0
    lens[B // 2] = 18
    s = Path(rs, B, 3, 1, 64)
    off, rows = np.cumsum([0, *lens]), int(lens.sum())
    kv = [dev(rs.standard_normal((rows, 64))).bfloat16() for _ in range(2)]
    P.dllava_mx_cache_store(kv[0], kv[1], 64, B, i32(off), i32(start), rows, None, None, s.cache, s.err, P.BF16)
    K, V = (f64(t).reshape(-1, 1, 64) for t in kv)
    for b in range(B):
        for i in range(lens[b]):
            s.ref.put(b, start[b] + i, K[off[b] + i], V[off[b] + i])
        s.ref.lens[b] = start[b] + lens[b]
    s.same()
    out = [torch.full_like(t, 9.0) for t in kv]
    P.dllava_mx_cache_load(s.cache, B, i32(off), i32(start), rows, *out, 64, P.BF16)
    for t, x in zip(out, (K, V)):
        assert np.array_equal(f64(t), R.dequantize(*R.quantize(x[:, 0])))


def test_store_of_nothing_sets_the_lengths():
    rs = np.random.default_rng(2)
    s = Path(rs, 3, 2, 1, 64)
    P.dllava_mx_cache_store(None, None, 64, 3, i32([0, 0, 0, 0]), i32([4, 0, 9]), 0, None, None, s.cache, s.err, P.F32)
    assert s.len.tolist() == [4, 0, 9]


# ---- the decode step ----------------------------------------------------------------------------------------------------------------
def step_and_check(s, rs, Hq, ws, keep=None, threshold=0.25, scale=None):
    """One step on the device and in the oracle; every output is compared."""
    B, H, Dh = s.B, s.H, s.Dh
    scale = Dh ** -0.5 if scale is None else scale
    q = dev(rs.standard_normal((B, Hq, Dh)) * 2).bfloat16()
    k, v = (dev(rs.standard_normal((B, H, Dh))).bfloat16() for _ in range(2))
    logits = dev(rs.standard_normal((B, 2)).astype(np.float32))
    o, keep_out = torch.full_like(q, float("nan")), torch.full((B,), 77, dtype=torch.uint8, device=DEV)
    P.dllava_mx_decode_attn_append(q, k, v, B, Hq, logits, threshold, None if keep is None else dev(np.asarray(keep, np.uint8)), s.cache, scale, o,
                                   keep_out, s.err, ws)
    lg = logits.cpu().numpy()
    kept = (lg[:, 1] - lg[:, 0] > np.float32(threshold)) if keep is None else np.asarray(keep) != 0
    for b in range(B):
        n = int(s.ref.lens[b])
        K, V = s.ref.rows(b, n)
        K, V = np.concatenate([K, f64(k[b:b + 1])]), np.concatenate([V, f64(v[b:b + 1])])
        want, W, A = (t[0] for t in R.attention(f64(q[b:b + 1]), K, V, scale))
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2 * (Dh + 16) * 2.0 ** -23 * A[:, None] + 2 * (n + 1) * 2.0 ** -23) * W
        bad = ~(np.abs(f64(o[b]) - want) <= tol)
        assert not bad.any(), (b, n, bad.sum(), np.argwhere(bad)[:4], np.nanmax(np.abs(f64(o[b]) - want)))
        if kept[b] and n < s.cap:
            s.ref.put(b, n, f64(k[b]), f64(v[b]))
            s.ref.lens[b] += 1
    assert np.array_equal(keep_out.cpu().numpy(), kept.astype(np.uint8))
    s.same()
    assert (ws[:256 * B] == 0).all()                        # the sequences' counters are back at zero


def workspace(s, Hq):
    return torch.zeros(P.dllava_mx_decode_workspace(s.B, Hq, s.H, s.Dh, s.cache.max_pages_per_seq), dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("splits", [0, 1, 2, 5])
@pytest.mark.parametrize("H,G,Dh", [(1, 1, 64), (2, 4, 128), (3, 7, 64), (2, 1, 128), (1, 16, 128), (2, 17, 64), (1, 32, 128), (5, 2, 64)])
def test_decode_steps(H, G, Dh, splits):
    rs = np.random.default_rng(H * G + Dh)
    lens = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 200]
    s = Path(rs, len(lens), 15, H, Dh)
    s.fill(rs, lens)
    ws = workspace(s, H * G)
    P.dllava_set_launch_override(P.LAUNCH_DECODE_SPLITS, splits)
    try:
        for _ in range(3):
            step_and_check(s, rs, H * G, ws)
    finally:
        P.dllava_set_launch_override(P.LAUNCH_DECODE_SPLITS, 0)
    assert int(s.err) == 0


def test_decode_long_sequence():
    rs = np.random.default_rng(8)
    s = Path(rs, 2, 190, 2, 128)
    s.fill(rs, [3001, 7])
    ws = workspace(s, 8)
    step_and_check(s, rs, 8, ws, keep=[1, 1])
    step_and_check(s, rs, 8, ws, keep=[0, 1], scale=1.0)     # sharp softmax: the reference moves


@pytest.mark.parametrize("splits", [0, 1, 7])
@pytest.mark.parametrize("B,H,G,Dh", [(70, 2, 2, 64), (300, 2, 1, 64), (130, 5, 17, 64)])
def test_decode_many_sequences(B, H, G, Dh, splits):
    """More sequences than lanes, and units than blocks; lengths of zero to five steps."""
    rs = np.random.default_rng(B)
    s = Path(rs, B, 9, H, Dh)
    s.fill(rs, rs.choice([0, 0, 1, 2, 15, 16, 17, 33, 140], B))
    ws = workspace(s, H * G)
    P.dllava_set_launch_override(P.LAUNCH_DECODE_SPLITS, splits)
    try:
        for _ in range(2):
            step_and_check(s, rs, H * G, ws)
    finally:
        P.dllava_set_launch_override(P.LAUNCH_DECODE_SPLITS, 0)


@pytest.mark.parametrize("lens,H,G", [([20000], 1, 4), ([17, 12000, 9000], 1, 16), ([40, 20000, 0, 500], 1, 1), ([6000, 6100], 4, 2)])
def test_decode_units_of_many_blocks(lens, H, G):
    """Sequences long enough to be cut into up to 65 parts (H = 1: the fewest units), beside short ones."""
    rs = np.random.default_rng(sum(lens))
    s = Path(rs, len(lens), max(lens) // 16 + 1, H, 64)
    rows = sum(lens)
    k, v = (dev(rs.standard_normal((rows, H, 64))).bfloat16() for _ in range(2))
    P.dllava_mx_cache_store(k, v, H * 64, len(lens), i32(np.cumsum([0] + lens)), None, rows, None, None, s.cache, s.err, P.BF16)
    s.ref.pages, s.ref.lens = s.pages.cpu().numpy(), np.asarray(lens, np.int64)   # (the store's bytes are tested above)
    ws = workspace(s, H * G)
    for _ in range(2):
        step_and_check(s, rs, H * G, ws, keep=[1] * len(lens))


def test_decode_at_capacity():
    rs = np.random.default_rng(9)
    s = Path(rs, 3, 2, 2, 64)
    s.fill(rs, [31, 32, 5])
    ws = workspace(s, 4)
    step_and_check(s, rs, 4, ws, keep=[1, 0, 1])
    assert int(s.err) == 0
    step_and_check(s, rs, 4, ws, keep=[1, 0, 1])             # sequence 0 is full now
    assert int(s.err) == 1


def test_decode_growing_maxima():
    """Keys whose scores grow along the sequence: the reference of the exponentials moves again and again."""
    rs = np.random.default_rng(10)
    s = Path(rs, 1, 40, 1, 128)
    n = 600
    base = rs.standard_normal((1, 128))
    for t in range(n):
        s.ref.put(0, t, base * (t / 20.0) * (1 if t % 3 else -1), rs.standard_normal((1, 128)))
    s.ref.lens[0] = n
    s.pages.copy_(dev(s.ref.pages)), s.len.fill_(n)
    step_and_check(s, rs, 4, workspace(s, 4))


def test_decode_nan_stays_with_its_sequence_and_head():
    rs = np.random.default_rng(11)
    s = Path(rs, 2, 4, 2, 64)
    s.fill(rs, [40, 41])
    k = rs.standard_normal((2, 64))
    k[1, 5] = np.nan
    s.ref.put(0, 20, k, k)                                   # head 1 of sequence 0
    s.pages.copy_(dev(s.ref.pages))
    q = dev(rs.standard_normal((2, 4, 64))).bfloat16()
    kv = dev(rs.standard_normal((2, 2, 64))).bfloat16()
    o = torch.zeros_like(q)
    P.dllava_mx_decode_attn_append(q, kv, kv, 2, 4, None, 0.0, torch.zeros(2, dtype=torch.uint8, device=DEV), s.cache, 0.125, o, None, None, workspace(s, 4))
    nan = np.isnan(f64(o))
    assert nan[0, 2:, :32].all() and not nan[0, :2].any() and not nan[1].any()


def test_decode_one_workspace_for_calls_of_many_sizes():
    """A batch that shrinks and grows, other heads and other caches, on one workspace of the largest call's size."""
    rs = np.random.default_rng(15)
    paths = [(Path(rs, B, mp, H, Dh), Hq) for B, mp, H, Dh, Hq in ((1, 3, 1, 64, 4), (40, 40, 2, 64, 8), (3, 60, 4, 128, 4), (70, 5, 1, 64, 16))]
    for s, _ in paths:
        s.fill(rs, rs.integers(0, s.cap - 2, s.B))
    ws = torch.zeros(max(workspace(s, Hq).numel() for s, Hq in paths), dtype=torch.uint8, device=DEV)
    for i in (0, 1, 2, 1, 3, 0, 2):
        step_and_check(*paths[i][:1], rs, paths[i][1], ws)


def test_decode_captured_and_on_another_stream():
    rs = np.random.default_rng(12)
    s, t = Path(rs, 5, 8, 2, 128, junk=0), None
    s.fill(rs, [3, 0, 50, 64, 100])
    Hq = 8
    ws = workspace(s, Hq)
    q, k, v = (torch.zeros((5, h, 128), dtype=torch.bfloat16, device=DEV) for h in (Hq, 2, 2))
    keep, o = torch.ones(5, dtype=torch.uint8, device=DEV), torch.zeros((5, Hq, 128), dtype=torch.bfloat16, device=DEV)
    pages0, len0 = s.pages.clone(), s.len.clone()
    call = lambda: P.dllava_mx_decode_attn_append(q, k, v, 5, Hq, None, 0.0, keep, s.cache, 0.1, o, None, s.err, ws)
    tokens = [[dev(rs.standard_normal(x.shape)).bfloat16() for x in (q, k, v)] + [dev(rs.integers(0, 2, 5).astype(np.uint8))] for _ in range(4)]
    eager = []
    for tok in tokens:
        for a, b_ in zip((q, k, v, keep), tok):
            a.copy_(b_)
        call()
        eager.append(o.clone())
    pages1, len1 = s.pages.clone(), s.len.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    s.pages.copy_(pages0), s.len.copy_(len0)
    for tok, want in zip(tokens, eager):
        for a, b_ in zip((q, k, v, keep), tok):
            a.copy_(b_)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want)
    assert torch.equal(s.pages, pages1) and torch.equal(s.len, len1)
    s.pages.copy_(pages0), s.len.copy_(len0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for tok, want in zip(tokens, eager):
            for a, b_ in zip((q, k, v, keep), tok):
                a.copy_(b_)
            call()
            assert torch.equal(o, want)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(s.pages, pages1) and torch.equal(s.len, len1)


def test_decode_shares_pages_between_sequences():
    """Two sequences with the same first pages in their tables (a prompt answered twice) read the same keys."""
    rs = np.random.default_rng(13)
    s = Path(rs, 2, 6, 2, 64)
    s.fill(rs, [48, 48])
    table = s.ref.table.copy()
    table[1, :3] = table[0, :3]
    s.ref.table = table
    s.cache = P.KVCache(s.pages, dev(table), s.len)
    ws = workspace(s, 2)
    for _ in range(2):
        step_and_check(s, rs, 2, ws, keep=[1, 1])
