"""The paged 8-bit cache on the GPU against its definition in 64 bits (paged_reference): tables, slot maps, append, read-back,
single-token attention, chunks, and a serving loop of all of them."""
import math

import numpy as np
import pytest
import torch

from tests import paged_reference as R

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def lg():
    from paper_2410_01485_b200 import binding, build
    build.build()
    binding.load_library()
    return binding


def dev(x, dtype=None):
    return torch.as_tensor(x, dtype=dtype).cuda()


def np64(t):
    return t.detach().double().cpu().numpy()


class Setup:
    """A pool of random pages, a table over a permutation of them (every second sequence's pages backwards), and the same
    for the reference."""

    def __init__(self, lg, n, Hq, Hkv, D, sink, window, P, seed=0, extra=3, block=0, pad=0, scales=(-3, 3), num_pages=None):
        B, self.n, self.lg = len(n), list(n), lg
        cols = -(-(sink + window) // P)
        self.num_pages = num_pages or B * cols + extra
        rng = np.random.RandomState(seed)
        perm = rng.permutation(self.num_pages)[:B * cols].reshape(B, cols)
        perm[1::2] = perm[1::2, ::-1]
        table = np.full((B, cols + pad), -7, dtype=np.int32)
        table[:, :cols] = perm
        codes = [rng.randint(0, 127, (self.num_pages, Hkv, P, D)) | (rng.randint(0, 2, (self.num_pages, Hkv, P, D)) << 7) for _ in "kv"]
        # magnitudes as quantised activations have them: normal numbers over the page's scale
        x = [rng.randn(self.num_pages, Hkv, P, D) for _ in "kv"]
        scale = [2.0 ** rng.randint(scales[0], scales[1] + 1, (self.num_pages, Hkv)) / 128 for _ in "kv"]
        codes = [R.encode_e4m3(np.clip(v * 100, -440, 440)).astype(np.uint8) for v in x]
        self.p = lg.paged_params(B, Hq, Hkv, D, sink, window, page_tokens=P, num_pages=self.num_pages, block_tokens=block,
                                 table_stride=cols + pad if pad else 0)
        self.ref = R.Cache(sink, window, P, codes[0], codes[1], scale[0].astype(np.float32), scale[1].astype(np.float32), table)
        self.block = block
        self.upload()

    def upload(self):
        c = self.ref
        self.pools = [torch.from_numpy(x.copy()).cuda().view(F8) for x in c.codes]
        self.scales = [dev(s, torch.float32) for s in c.scale]
        self.table = dev(c.table, torch.int32)

    @property
    def cache(self):
        return (*self.pools, *self.scales)

    def counts(self, n=None):
        return dev(self.n if n is None else n, torch.int64)

    def same_state(self):
        for pool, scale, codes, want in zip(self.pools, self.scales, self.ref.codes, self.ref.scale):
            got = pool.view(torch.uint8).cpu().numpy()
            nan = (got & 127) == 127
            assert np.array_equal(nan, (codes & 127) == 127)
            assert np.array_equal(got[~nan], codes[~nan])
            assert np.array_equal(np64(scale), want)

    def check_decode(self, q, o, lse, n=None, q_scale=None):
        c, p = self.ref, self.p
        G = p.Hq // p.Hkv
        scale = p.scale or 1 / math.sqrt(p.D)
        q, o, lse = np64(q), np64(o), np64(lse)
        for b, nb in enumerate(self.n if n is None else n):
            for h in range(p.Hkv):
                pos, k, v = c.rows(b, h, nb)
                see = R.visible(nb - 1, pos, c.sink, c.window, self.block)
                # codes that are f16 weights below 2^-14 lose bits: 2^-25 of the largest weight each
                for g in range(h * G, h * G + G):
                    if see.any():
                        s = k[see] @ q[b, g] * scale
                        page = np.array([c.page(b, R.slot_of(int(j), c.sink, c.window)) for j in pos[see]])
                        vs = c.scale[1][page, h]
                        w = np.exp(s - s.max())
                        extra = 2.0 ** -25 * (w * vs).max() * np.abs(v[see] / vs[:, None]).sum(0) / w.sum()
                    else:
                        extra = 0.0
                    want, l, tol, tol_l = R.attend(q[b, g], k, v, see, scale, 2.0 ** -11, extra)
                    assert np.all(np.abs(o[b, g] - want) <= tol), (b, g, np.abs(o[b, g] - want).max(), tol.max())
                    assert (l == lse[b, g]) if math.isinf(l) else abs(lse[b, g] - l) <= tol_l, (b, g, l, lse[b, g], tol_l)


def randn(*shape, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g, device="cuda")).to(torch.bfloat16)


# ------------------------------------------------------------------------------- tables, slot maps

@pytest.mark.parametrize("B, T, sink, window, P, hi, pad", [
    (1, 1, 0, 50, 16, 60, 0), (5, 1, 64, 256, 64, 500, 3), (33, 7, 4, 1003, 16, 1500, 0), (300, 300, 0, 2000, 32, 2500, 1),
    (700, 5, 128, 4096, 64, 6000, 0), (2, 40000, 0, 40000, 16, 10, 0),
])
@pytest.mark.parametrize("counts", [True, False])
def test_table_extend(lg, B, T, sink, window, P, hi, pad, counts):
    rng = np.random.RandomState(B + T)
    n = rng.randint(0, hi + 1, B)
    n[rng.rand(B) < 0.2] = 0
    if B > 4:
        n[1], n[3] = -3, 1 << 40
    new = rng.randint(0, T + 1, B) if counts else np.full(B, T)
    if counts and B > 4:
        new[0], new[4] = -2, T + 50 if T < 40000 else T      # below and above the range: taken as 0 and T
    eff = np.clip(new, 0, T)
    cols = -(-(sink + window) // P)
    have = np.array([R.pages_of(int(x), sink, window, P) for x in n])
    need = np.array([have[b] if n[b] < 0 else R.pages_of(int(n[b]) + int(eff[b]), sink, window, P) for b in range(B)])
    wanted = int((need - have).sum())
    p = lg.paged_params(B, 8, 2, 128, sink, window, page_tokens=P, num_pages=1 << 17, table_stride=cols + pad if pad else 0)
    for n_free, start in ((wanted + 9, 4), (max(1, wanted // 2 + 3), 3)):
        free = rng.permutation(1 << 17)[:n_free].astype(np.int32)
        table = rng.randint(-5, 5, (B, cols + pad)).astype(np.int32)
        want, at = table.copy(), start
        for b in range(B):
            for i in range(have[b], need[b]):
                want[b, i] = free[at] if at < n_free else -1
                at += 1
        t, nxt = dev(table, torch.int32), dev([-1], torch.int32)
        for _ in range(2):                                    # repeating the call changes nothing
            lg.lg_paged_table_extend(p, dev(n, torch.int64), dev(new, torch.int32) if counts else None, dev(free, torch.int32),
                                     dev([start], torch.int32), t, nxt, T_new=T)
            assert np.array_equal(t.cpu().numpy(), want) and nxt.item() == at


@pytest.mark.parametrize("B, T, sink, window, P", [(1, 1, 0, 50, 16), (3, 500, 64, 256, 64), (4, 1300, 5, 1003, 16), (40, 9, 0, 77, 128)])
def test_slot_map(lg, B, T, sink, window, P):
    rng = np.random.RandomState(T)
    cols = -(-(sink + window) // P)
    table = rng.permutation(4096)[:B * cols].reshape(B, cols).astype(np.int32)
    table[rng.rand(B, cols) < 0.1] = -1
    table[0, 0] = 4096                                         # names no page of the pool
    n = rng.randint(0, 2 * (sink + window), B)
    n[-1] = sink + window + (1 << 41)
    first = np.maximum(0, n - rng.randint(0, T + 40, B))
    first[0] = -3
    count = rng.randint(0, T + 1, B)
    p = lg.paged_params(B, 4, 4, 64, sink, window, page_tokens=P, num_pages=4096)
    for cnt in (count, None):
        want = np.full((B, T), -1, dtype=np.int64)
        for b in range(B):
            held = {j: s for s, j in R.ring(int(n[b]), sink, window).items()}
            for t in range(T if cnt is None else cnt[b]):
                s = held.get(int(first[b]) + t)
                if s is not None and 0 <= table[b, s // P] < 4096:
                    want[b, t] = table[b, s // P] * P + s % P
        out = torch.full((B, T), 77, dtype=torch.int64, device="cuda")
        lg.lg_paged_slot_map(p, dev(n, torch.int64), dev(first, torch.int64), None if cnt is None else dev(cnt, torch.int32),
                             dev(table, torch.int32), out)
        assert np.array_equal(out.cpu().numpy(), want)


# ---------------------------------------------------------------------------------- append, gather

APPENDS = [  # n, T, new, Hkv, D, sink, window, P
    ([0], 1, None, 1, 128, 0, 40, 16),
    ([5, 63, 64, 700], 1, None, 2, 128, 64, 128, 64),
    ([3, 0, 250], 37, None, 2, 64, 4, 203, 16),
    ([0, 100, 31], 150, [150, 0, 77], 3, 128, 64, 192, 32),
    ([17, 1 << 40], 1000, [999, 1000], 1, 64, 0, 333, 128),
    ([0, 90], 777, None, 1, 128, 10, 300, 128),
    ([200, -1, 10], 2, [2, 2, -4], 2, 64, 0, 96, 64),
    ([200, -1, 10, 0, 1 << 40], 1, [1, 1, 0, 3, 1], 2, 128, 5, 203, 128),
    ([7, 0, 63, 64, 100], 1, [0, 1, 1, -2, 1], 3, 64, 0, 64, 16),
]


@pytest.mark.parametrize("case", APPENDS, ids=lambda c: "n%s_T%d_D%d_P%d" % (c[0][0], c[1], c[4], c[7]))
@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
def test_append(lg, case, layout):
    n, T, new, Hkv, D, sink, window, P = case
    s = Setup(lg, n, Hkv, Hkv, D, sink, window, P, seed=T, pad=2)
    rng = np.random.RandomState(T)
    rows = []
    for seed in (1, 2):
        x = randn(len(n), Hkv, T, D, seed=seed) * dev(2.0 ** rng.randint(-6, 7, (len(n), Hkv, T, 1)), torch.bfloat16)
        rows.append(x if layout == "bhtd" else x.transpose(1, 2).contiguous().transpose(1, 2))
    count = None if new is None else dev(new, torch.int32)
    lg.lg_paged_append(s.p, *s.cache, s.table, *rows, s.counts(), count)
    k, v = (np64(x) for x in rows)
    for b, nb in enumerate(n):
        t = T if new is None else max(0, new[b])
        s.ref.append(b, nb, k[b, :, :t], v[b, :, :t])
    s.same_state()
    lg.lg_paged_append(s.p, *s.cache, s.table, *rows, s.counts(), count)     # the same tokens over themselves
    s.same_state()


def test_append_grows_and_shrinks_scales(lg):
    """A large token raises its page's scale (the others' codes move, small ones round), and the scale falls when the ring
    has overwritten it; zeros, infinities and NaN."""
    s = Setup(lg, [0, 0], 2, 2, 64, 0, 32, 16)
    size = [1.0, 1e-3, 300.0, 1e5, 1e-4, 3e38, 0.0, 1e-38] + [1.0] * 40
    for j, m in enumerate(size):
        k, v = randn(2, 2, 1, 64, seed=j) * m, randn(2, 2, 1, 64, seed=100 + j) * m
        if j in (2, 20):
            k[0, 1, 0, 5], v[0, 0, 0, 7], v[1, 1, 0, 0] = float("inf"), float("nan"), -float("inf")
        if j == 9:
            k[0, 0] = float("nan")
        lg.lg_paged_append(s.p, *s.cache, s.table, k, v, s.counts([j, j]))
        for b in range(2):
            s.ref.append(b, j, np64(k)[b], np64(v)[b])
        s.same_state()


@pytest.mark.parametrize("T", [1, 40])
def test_append_bad_pages_and_neighbours(lg, T):
    """Table entries that name no page: their tokens are dropped, nothing else is touched."""
    s = Setup(lg, [64, 3, 90], 2, 2, 128, 0, 96, 32)
    s.ref.table[0, 2] = -1
    s.ref.table[1, 0] = s.num_pages
    s.ref.table[2, :] = np.iinfo(np.int32).max
    s.upload()
    k, v = randn(3, 2, T, 128, seed=1), randn(3, 2, T, 128, seed=2)
    lg.lg_paged_append(s.p, *s.cache, s.table, k, v, s.counts())
    for b in range(3):
        s.ref.append(b, s.n[b], np64(k)[b], np64(v)[b])
    s.same_state()


@pytest.mark.parametrize("D, P, T", [(128, 64, 1), (64, 16, 333), (128, 16, 50), (64, 128, 7)])
def test_gather(lg, D, P, T):
    s = Setup(lg, [1] * 3, 2, 2, D, 0, 300, P, scales=(-40, 40))
    rng = np.random.RandomState(T)
    top = s.num_pages * P
    slots = rng.randint(0, top, (3, T))
    slots[:, 0] = slots[0, 0]                                   # the same row several times
    if T > 5:
        slots[0, 1], slots[1, 2], slots[2, 3], slots[1, 4] = -1, top, -(1 << 40), 1 << 50
    k, v = lg.lg_paged_gather(s.p, *s.cache, dev(slots, torch.int64))
    ok = (slots >= 0) & (slots < top)
    at = np.where(ok, slots, 0)
    for got, codes, scale in zip((k, v), s.ref.codes, s.ref.scale):
        want = R.decode_e4m3(codes[at // P, :, at % P]) * scale[at // P][..., None]
        assert np.array_equal(np64(got), np.where(ok[..., None, None], want, 0.0).transpose(0, 2, 1, 3))


# ------------------------------------------------------------------------------ single-token attention

DECODES = [  # n, Hq, Hkv, D, sink, window, P, block
    ([1], 1, 1, 128, 0, 16, 16, 0),
    ([0, 1, 15, 16, 17, 31, 32, 33], 8, 1, 128, 0, 300, 16, 0),
    ([200, 0, 330, 64], 12, 4, 64, 64, 256, 64, 0),
    ([131072, 5, 2000], 64, 8, 128, 128, 1024, 64, 0),
    ([3000, 700, 1 << 40], 16, 1, 64, 4, 1003, 32, 0),
    ([999, 130, 64, 65], 24, 2, 128, 64, 256, 128, 64),
    ([700, 450, 100], 6, 2, 64, 0, 192, 16, 32),
    ([4000, 3999], 2, 2, 128, 0, 4096, 16, 0),
]


@pytest.mark.parametrize("case", DECODES, ids=lambda c: "n%d_%d_%d_D%d_P%d" % (c[0][0], c[1], c[2], c[3], c[6]))
def test_decode(lg, case):
    n, Hq, Hkv, D, sink, window, P, block = case
    s = Setup(lg, n, Hq, Hkv, D, sink, window, P, block=block, pad=1)
    q = randn(len(n), Hq, D, seed=3)
    ws = lg.paged_decode_workspace(s.p)
    o, lse = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts(), workspace=ws)
    s.check_decode(q, o, lse)
    again, lse2 = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts(), workspace=ws)
    assert torch.equal(o, again) and torch.equal(lse, lse2) and lg.lg_last_status(ws) == 0
    only, none = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts(), workspace=ws, want_lse=False)
    assert none is None and torch.equal(o, only)


SLICES = [  # n, Hq, Hkv, D, window, P: how units (sequence, kv head) and CTAs share each other
    ([900, 0, 33, 2000], 8, 1, 128, 2048, 16),                    # several CTAs a unit, of unequal lengths
    ([0, 0, 1, 5000], 6, 3, 64, 4096, 64),
    ([500 + b if b % 9 else 0 for b in range(40)], 8, 4, 64, 512, 32),   # one CTA a unit, sequences beyond the first 32
    ([97 + b % 31 for b in range(40)], 8, 8, 128, 128, 16),       # three units a CTA, all of four tiles
    ([97] * 39 + [96], 8, 8, 128, 128, 16),                       # ... and one of three
    ([8000] + [10] * 20, 4, 4, 128, 8192, 128),                   # across units: one of them is far longer than the rest
    ([300] * 299, 1, 1, 64, 288, 32),                             # more sequences than are looked at
]


@pytest.mark.parametrize("case", SLICES, ids=lambda c: "B%d_%d_%d_D%d_W%d" % (len(c[0]), c[1], c[2], c[3], c[4]))
def test_decode_slices(lg, case):
    n, Hq, Hkv, D, window, P = case
    s = Setup(lg, n, Hq, Hkv, D, 0, window, P)
    q = randn(len(n), Hq, D, seed=3)
    ws = lg.paged_decode_workspace(s.p)
    ws[256 + 4 * len(n) * Hkv + 256:] = 255                       # records that are read have been written
    o, lse = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts(), workspace=ws)
    s.check_decode(q, o, lse)
    again, lse2 = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts(), workspace=ws)
    assert torch.equal(o, again) and torch.equal(lse, lse2) and lg.lg_last_status(ws) == 0


@pytest.mark.parametrize("D, P, block", [(128, 16, 0), (64, 64, 32), (128, 32, 32)])
def test_decode_reads_nothing_it_does_not_attend(lg, D, P, block):
    """NaN codes and NaN scales in empty slots, in pages of nobody, and in ring tokens that the block-aligned window leaves out."""
    n = [0, 1, 20, 95, 200]
    s = Setup(lg, n, 8, 2, D, 32, 96, P, block=block)
    q = randn(len(n), 8, D, seed=3)
    clean = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts())
    used = set()
    for b, nb in enumerate(n):
        for slot, j in R.ring(nb, 32, 96).items():
            if R.visible(nb - 1, np.array([j]), 32, 96, block)[0]:
                used.add((s.ref.page(b, slot), slot % P))
    for page in range(s.num_pages):
        for off in range(P):
            if (page, off) not in used:
                for x in range(2):
                    s.ref.codes[x][page, :, off] = 127
        if not any(u[0] == page for u in used):
            for x in range(2):
                s.ref.scale[x][page] = np.nan
    s.upload()
    o, lse = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts())
    assert torch.equal(o, clean[0]) and torch.equal(lse, clean[1])
    s.check_decode(q, o, lse)


@pytest.mark.parametrize("P, D", [(16, 128), (32, 64), (64, 128)])
def test_decode_pages_of_far_apart_scales(lg, P, D):
    """Neighbouring pages whose scales differ by up to 2^80: weights and sums keep their own references."""
    s = Setup(lg, [500, 77, 256], 4, 2, D, 0, 512, P, scales=(-40, 40))
    s.ref.scale[0][:] = 2.0 ** np.random.RandomState(1).randint(-9, -5, s.ref.scale[0].shape)
    s.upload()
    q = randn(3, 4, D, seed=5)
    o, lse = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts())
    s.check_decode(q, o, lse)
    # a scale that is no power of two, and one page dominating by its scores
    s.ref.scale[1][:] = s.ref.scale[1] * 1.3
    s.ref.scale[1] = s.ref.scale[1].astype(np.float32).astype(np.float64)
    s.upload()
    o, lse = lg.lg_paged_decode(s.p, 20 * q, *s.cache, s.table, s.counts())
    s.check_decode(20 * q, o, lse)


@pytest.mark.parametrize("P, D, spread, size", [(32, 64, 40, 20), (16, 128, 40, 20), (64, 64, 5, 5), (128, 128, 3, 5), (32, 64, 8, 20)])
def test_decode_long_runs_over_scales_and_scores_far_apart(lg, P, D, spread, size):
    """A warp works several tiles, whose scores and V scales rise and fall past each other."""
    n = [1024 - 7 * b for b in range(40)]
    s = Setup(lg, n, 4, 4, D, 0, 1024, P, scales=(-spread, spread))
    s.ref.scale[0][:] = 2.0 ** np.random.RandomState(1).randint(-9, -5, s.ref.scale[0].shape)
    s.upload()
    q = size * randn(40, 4, D, seed=5)
    o, lse = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts())
    s.check_decode(q, o, lse)


@pytest.mark.parametrize("m", [2.0 ** -100, 2.0 ** 60, 0.0])
def test_decode_q_of_any_size(lg, m):
    s = Setup(lg, [100, 300], 4, 1, 128, 0, 512, 32)
    s.ref.scale[0][:] = 1.0 / 64 if m == 0 else min(2.0 ** 100, 1 / m) / 64
    s.upload()
    q = randn(2, 4, 128, seed=5) * m
    o, lse = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts())
    s.check_decode(q, o, lse)


def test_decode_absent_pages_are_reported_and_left_out(lg):
    s = Setup(lg, [100, 300, 40], 8, 2, 128, 0, 320, 16)
    s.ref.table[0, 2] = -1
    s.ref.table[1, 5:9] = s.num_pages + 3
    s.ref.table[2, :] = -1                                       # nothing is left of this one
    s.upload()
    q = randn(3, 8, 128, seed=5)
    ws = lg.paged_decode_workspace(s.p)
    o, lse = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts(), workspace=ws)
    s.check_decode(q, o, lse)
    assert lg.lg_last_status(ws) == -7 and lg.lg_last_status(ws) == 0
    assert torch.isinf(lse[2]).all() and not o[2].any()


@pytest.mark.parametrize("where", ["k", "v", "q"])
def test_decode_nan_that_is_attended_stays(lg, where):
    """... in the heads that read it, and only there; in a run of its own, a shared unit and a CTA's piece."""
    s = Setup(lg, [2000, 40, 33], 4, 2, 128, 0, 2048, 16)
    q = randn(3, 4, 128, seed=5)
    clean = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts())
    for b in range(3):
        if where == "q":
            q[b, 2, 5] = float("nan")
        else:
            s.ref.codes[where == "v"][s.ref.page(b, 30), 1, 30 % 16, 7] = 127
    s.upload()
    o, lse = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts())
    hit = torch.zeros(4, dtype=torch.bool, device="cuda")
    hit[2:3 if where == "q" else 4] = True
    assert torch.equal(o[:, ~hit], clean[0][:, ~hit]) and torch.equal(lse[:, ~hit], clean[1][:, ~hit])
    if where == "v":
        assert torch.isnan(o[:, hit, 7]).all() and torch.equal(lse, clean[1])
        o[:, hit, 7] = clean[0][:, hit, 7]
        assert torch.equal(o, clean[0])
    else:
        assert torch.isnan(o[:, hit]).all() and torch.isnan(lse[:, hit]).all()


def test_decode_shared_pages_and_scale(lg):
    """Two sequences read the same pages (a shared prompt); a softmax scale of one's own."""
    s = Setup(lg, [90, 200, 90], 4, 2, 64, 0, 256, 16)
    s.ref.table[2] = s.ref.table[0]
    s.p.scale = 0.31
    s.upload()
    q = randn(3, 4, 64, seed=5)
    q[2] = q[0]
    o, lse = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts())
    s.check_decode(q, o, lse)
    assert (o[0].float() - o[2].float()).abs().max() <= 2.0 ** -7 * o[0].float().abs().max()


def test_decode_many_sequences(lg):
    """More sequences than one launch takes, most of them empty or short."""
    B = 4096 + 37
    n = [(7 * b) % 19 for b in range(B)]
    s = Setup(lg, n, 2, 1, 64, 0, 32, 16, num_pages=2 * B)
    q = randn(B, 2, 64, seed=5)
    o, lse = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts())
    s.check_decode(q, o, lse)


def test_offsets_beyond_32_bits(lg):
    """A pool of more than 2^32 bytes: append, read-back and attention at its far end."""
    P, Hkv, D = 64, 8, 128
    num = (1 << 32) // (P * Hkv * D) + 70
    pool = torch.zeros(num, Hkv, P, D, dtype=torch.uint8, device="cuda").view(F8)
    scale = torch.ones(num, Hkv, device="cuda")
    p = lg.paged_params(1, 8, Hkv, D, 0, 256, page_tokens=P, num_pages=num)
    small = lg.paged_params(1, 8, Hkv, D, 0, 256, page_tokens=P, num_pages=4)
    far, near = dev([[num - 1, 0, num - 60, num - 2]], torch.int32), dev([[3, 0, 1, 2]], torch.int32)
    k, v, q = randn(1, Hkv, 250, D, seed=1), randn(1, Hkv, 250, D, seed=2), randn(1, 8, D, seed=3)
    sp = [torch.zeros(4, Hkv, P, D, dtype=torch.uint8, device="cuda").view(F8) for _ in "kv"]
    ss = [torch.ones(4, Hkv, device="cuda") for _ in "kv"]
    n0, n1 = dev([0], torch.int64), dev([250], torch.int64)
    v_pool, v_scale = pool.clone(), scale.clone()
    lg.lg_paged_append(p, pool, v_pool, scale, v_scale, far, k, v, n0)
    lg.lg_paged_append(small, *sp, *ss, near, k, v, n0)
    a = lg.lg_paged_decode(p, q, pool, v_pool, scale, v_scale, far, n1)
    b = lg.lg_paged_decode(small, q, *sp, *ss, near, n1)
    maps = [torch.empty(1, 250, dtype=torch.int64, device="cuda") for _ in "ab"]
    lg.lg_paged_slot_map(p, n1, n0, None, far, maps[0])
    lg.lg_paged_slot_map(small, n1, n0, None, near, maps[1])
    x = lg.lg_paged_gather(p, pool, v_pool, scale, v_scale, maps[0])
    y = lg.lg_paged_gather(small, *sp, *ss, maps[1])
    for s, t in zip(a + x, b + y):
        assert torch.equal(s, t)
    assert x[0].float().abs().max() > 1


# ---------------------------------------------------------------------------------------- chunks

CHUNKS = [  # n, T, Hq, Hkv, D, sink, window, P, block
    ([0], 1, 2, 1, 128, 0, 64, 16, 0),
    ([0, 0], 100, 4, 2, 64, 64, 128, 32, 0),
    ([150, 150, 1000, 33], 77, 4, 2, 128, 64, 256, 64, 0),
    ([500, 731, 4000], 130, 2, 1, 64, 64, 192, 128, 0),
    ([500, 531, 564, 20], 61, 4, 1, 128, 64, 192, 16, 32),
]


@pytest.mark.parametrize("case", CHUNKS, ids=lambda c: "n%d_T%d_D%d_P%d" % (c[0][0], c[1], c[4], c[7]))
def test_chunk(lg, case):
    n, T, Hq, Hkv, D, sink, window, P, block = case
    B, G = len(n), Hq // Hkv
    s = Setup(lg, n, Hq, Hkv, D, sink, window, P, block=block, pad=1)
    for b, nb in enumerate(n):                                    # entries of pages without tokens are not read
        s.ref.table[b, R.pages_of(nb, sink, window, P):] = -1
    s.upload()
    q, k, v = randn(B, Hq, T, D, seed=1), randn(B, Hkv, T, D, seed=2), randn(B, Hkv, T, D, seed=3)
    ws = lg.paged_chunk_prefill_workspace(s.p, T, n)
    o, lse = lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n, workspace=ws)
    assert lg.lg_last_status(ws) == 0
    qd, kd, vd, od, ld = (np64(x) for x in (q, k, v, o, lse))
    for b, nb in enumerate(n):
        for h in range(Hkv):
            pos, ck, cv = s.ref.rows(b, h, nb)
            pos = np.concatenate([pos, np.arange(nb, nb + T)])
            ck, cv = np.concatenate([ck, kd[b, h]]), np.concatenate([cv, vd[b, h]])
            for t in range(T):
                see = R.visible(nb + t, pos, sink, window, block)
                for g in range(h * G, h * G + G):
                    want, l, tol, tol_l = R.attend(qd[b, g, t], ck, cv, see, 1 / math.sqrt(D), 2.0 ** -8)
                    assert np.all(np.abs(od[b, g, t] - want) <= tol) and abs(ld[b, g, t] - l) <= tol_l, (b, g, t)
    again = lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n, workspace=ws)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


def _check_chunk_rows(s, n, T, q, k, v, o, lse, rows, heads, weight=2.0 ** -8):
    p, c = s.p, s.ref
    G = p.Hq // p.Hkv
    for b in range(len(n)):
        for g in heads:
            h = g // G
            pos, ck, cv = c.rows(b, h, n[b])
            pos = np.concatenate([pos, np.arange(n[b], n[b] + T)])
            ck, cv = np.concatenate([ck, np64(k[b, h])]), np.concatenate([cv, np64(v[b, h])])
            for t in rows:
                see = R.visible(n[b] + t, pos, c.sink, c.window, s.block)
                want, l, tol, tol_l = R.attend(np64(q[b, g, t]), ck, cv, see, 1 / math.sqrt(p.D), weight)
                assert np.all(np.abs(np64(o[b, g, t]) - want) <= tol) and abs(lse[b, g, t].item() - l) <= tol_l, (b, g, t)


RAGGED = [  # n, T, Hq, Hkv, D, sink, window, P, block: sequences that hold unequal numbers of tokens
    ([0, 5, 63, 64, 65, 190, 1000], 70, 2, 1, 64, 64, 128, 16, 0),
    ([0, 5, 63, 64, 65, 190, 1000], 65, 2, 1, 64, 64, 128, 32, 64),
    ([1, 0, 7], 5, 2, 2, 128, 64, 64, 16, 0),                     # none has its sink
    ([10, 100, 3, 400, 399], 200, 2, 1, 64, 64, 128, 64, 0),      # a chunk longer than the window, sinks that are not full
    ([0, 300, 90, 1], 90, 2, 1, 128, 0, 256, 128, 0),             # no sink
    ([130, 3000, 700, 129], 33, 2, 1, 128, 128, 2048, 64, 0),     # tiles cut along their keys, lists of unequal length
    ([70, 2500, 300], 257, 8, 2, 64, 64, 1024, 16, 0),
]


@pytest.mark.parametrize("case", RAGGED, ids=lambda c: "B%d_T%d_D%d_W%d_%d" % (len(c[0]), c[1], c[4], c[6], c[8]))
def test_chunk_of_sequences_at_their_own_positions(lg, case):
    n, T, Hq, Hkv, D, sink, window, P, block = case
    B = len(n)
    s = Setup(lg, n, Hq, Hkv, D, sink, window, P, block=block)
    for b, nb in enumerate(n):                                    # entries of pages without tokens are not read
        s.ref.table[b, R.pages_of(nb, sink, window, P):] = -1
    s.upload()
    q, k, v = randn(B, Hq, T, D, seed=1), randn(B, Hkv, T, D, seed=2), randn(B, Hkv, T, D, seed=3)
    ws = lg.paged_chunk_prefill_workspace(s.p, T, n)
    ws[256:] = 255                                                # NaN wherever the call reads what it has not written
    o, lse = lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n, workspace=ws)
    assert lg.lg_last_status(ws) == 0
    rows = sorted({0, 1, T // 3, T // 2, T - 2, T - 1} & set(range(T)))
    _check_chunk_rows(s, n, T, q, k, v, o, lse, rows, range(0, Hq, max(1, Hq // 2)))
    alone = [lg.lg_paged_chunk_prefill(lg.paged_params(1, Hq, Hkv, D, sink, window, page_tokens=P, num_pages=s.num_pages, block_tokens=block),
                                       q[b:b + 1], k[b:b + 1], v[b:b + 1], *s.cache, s.table[b:b + 1], [n[b]]) for b in range(B)]
    # every row against a call of its own: both are off by half a step of every weight and of o (2^-8 each), a score by 2^-19 scale sum |q k|
    size = [max(x.float().abs().max().item(), (np.abs(R.decode_e4m3(c)).max(axis=(2, 3)) * sc).max())
            for x, c, sc in zip((k, v), s.ref.codes, s.ref.scale)]
    tol_l = 2 * 2.0 ** -19 / math.sqrt(D) * D * q.float().abs().max().item() * size[0] + 2.0 ** -16
    for b in range(B):
        want = alone[b][0][0].float()
        assert ((o[b].float() - want).abs() <= 2 * (2.0 ** -8 + tol_l) * size[1] + 2 * 2.0 ** -8 * want.abs()).all()
        assert (lse[b] - alone[b][1][0]).abs().max() <= tol_l
    bad = next(b for b in range(B) if n[b] > 0)                   # an absent page of one sequence
    s.ref.table[bad, 0] = s.num_pages
    s.upload()
    lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n, workspace=ws)
    assert lg.lg_last_status(ws) == -7


def test_chunk_of_more_rows_than_one_block_schedules(lg):
    T, n = 17000, [90]                                            # 67 super-tiles
    s = Setup(lg, n, 2, 1, 64, 0, 128, 64)
    q, k, v = randn(1, 2, T, 64, seed=1), randn(1, 1, T, 64, seed=2), randn(1, 1, T, 64, seed=3)
    ws = lg.paged_chunk_prefill_workspace(s.p, T, n)
    o, lse = lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n, workspace=ws)
    assert lg.lg_last_status(ws) == 0
    _check_chunk_rows(s, n, T, q, k, v, o, lse, [0, 1, 37, 38, 255, 256, 9999, 16639, 16640, T - 1], [0, 1])


def test_chunk_of_many_rows_at_two_phases(lg):
    """One schedule for all sequences, which hold as many tokens but whose window's blocks lie differently."""
    T, n = 16400, [1000, 1030]                                    # 65 super-tiles
    s = Setup(lg, n, 1, 1, 64, 64, 128, 64, block=64)
    q, k, v = randn(2, 1, T, 64, seed=1), randn(2, 1, T, 64, seed=2), randn(2, 1, T, 64, seed=3)
    ws = lg.paged_chunk_prefill_workspace(s.p, T, n)
    o, lse = lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n, workspace=ws)
    assert lg.lg_last_status(ws) == 0
    _check_chunk_rows(s, n, T, q, k, v, o, lse, [0, 1, 23, 24, 25, 127, 128, 9999, T - 1], [0])


def test_chunk_of_two_tiles_an_sm_over_gaps(lg):
    """D = 64 on a grid whose CTAs share SMs, sequences that hold unequal numbers of tokens."""
    T, n = 300, [0, 31, 64, 100, 200, 319, 320, 5000]
    s = Setup(lg, n, 16, 4, 64, 64, 256, 32)
    q, k, v = randn(8, 16, T, 64, seed=1), randn(8, 4, T, 64, seed=2), randn(8, 4, T, 64, seed=3)
    ws = lg.paged_chunk_prefill_workspace(s.p, T, n)
    ws[256:] = 255
    o, lse = lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n, workspace=ws)
    assert lg.lg_last_status(ws) == 0
    _check_chunk_rows(s, n, T, q, k, v, o, lse, [0, 1, 63, 64, 127, 128, 255, 256, 299], [0, 7, 15])


def test_chunk_of_more_sequences_than_one_launch(lg):
    B, T = 133, 3
    n = [70 + b for b in range(B)]                                # full rings: one run of neighbours, each at its own offset
    n[131] = 5
    s = Setup(lg, n, 1, 1, 64, 0, 64, 16)
    q, k, v = randn(B, 1, T, 64, seed=1), randn(B, 1, T, 64, seed=2), randn(B, 1, T, 64, seed=3)
    ws = lg.paged_chunk_prefill_workspace(s.p, T, n)
    o, lse = lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n, workspace=ws)
    assert lg.lg_last_status(ws) == 0
    _check_chunk_rows(s, n, T, q, k, v, o, lse, range(T), [0])
    s.ref.table[130, 2] = -1                                      # found by the launch that starts behind the first 128
    s.upload()
    lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n, workspace=ws)
    assert lg.lg_last_status(ws) == -7


@pytest.mark.parametrize("D, Hq", [(128, 4), (64, 2)])
def test_chunk_over_keys_that_raise_the_maximum(lg, D, Hq):
    """Tokens far above the ones before them, again and again: references that move late, by a lot, and not at all."""
    n, T = [400], 300
    s = Setup(lg, n, Hq, 1, D, 64, 256, 32, scales=(0, 0))
    q, k, v = randn(1, Hq, T, D, seed=1), randn(1, 1, T, D, seed=2), randn(1, 1, T, D, seed=3)
    big = torch.ones(T, 1, device="cuda")
    big[torch.arange(0, T, 37)] = 6.0
    big[150], big[200] = 20.0, 40.0                               # scores in the hundreds: past 2^40 of what came before
    k = (k.float() * big).to(torch.bfloat16)
    o, lse = lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n)
    _check_chunk_rows(s, n, T, q, k, v, o, lse, range(0, T, 7), range(Hq))


@pytest.mark.parametrize("block", [0, 64])
def test_chunk_reads_nothing_that_no_row_sees(lg, block):
    """NaN in the ring's tokens that have left the window of the chunk's first row, in stale pages and empty slots."""
    n, T = [400, 1000, 120], 40
    s = Setup(lg, n, 2, 1, 64, 64, 128, 32, block=block)
    q, k, v = randn(3, 2, T, 64, seed=1), randn(3, 1, T, 64, seed=2), randn(3, 1, T, 64, seed=3)
    clean = lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n)
    used = {(s.ref.page(b, slot), slot % 32) for b in range(3) for slot, j in R.ring(n[b], 64, 128).items()
            if any(R.visible(n[b] + t, np.array([j]), 64, 128, block)[0] for t in range(T))}
    for page in range(s.num_pages):
        for off in range(32):
            if (page, off) not in used:
                s.ref.codes[0][page, :, off] = s.ref.codes[1][page, :, off] = 127
    s.upload()
    o, lse = lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n)
    assert torch.equal(o, clean[0]) and torch.equal(lse, clean[1])


def test_chunk_absent_page_is_reported_and_writes_nothing(lg):
    s = Setup(lg, [100], 2, 1, 128, 64, 128, 16)
    s.ref.table[0, 3] = -1
    s.upload()
    q, k, v = randn(1, 2, 9, 128, seed=1), randn(1, 1, 9, 128, seed=2), randn(1, 1, 9, 128, seed=3)
    o, lse = torch.full_like(q, 7.0), torch.full((1, 2, 9), 7.0, device="cuda")
    ws = lg.paged_chunk_prefill_workspace(s.p, 9, [100])
    lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, [100], o=o, lse=lse, workspace=ws)
    assert lg.lg_last_status(ws) == -7
    assert (o == 7).all() and (lse == 7).all()
    lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, [40], o=o, lse=lse, workspace=ws)   # does not reach the page
    assert lg.lg_last_status(ws) == 0 and not (o == 7).any()


# --------------------------------------------------------------------------------------- together

def _serve(lg, s, steps, T0, graph=False):
    """Prompts of T0[b] tokens, then `steps` single tokens: pages from the free list, append, attention; everything checked."""
    p, c, B = s.p, s.ref, len(s.n)
    free = dev(np.random.RandomState(9).permutation(s.num_pages), torch.int32)
    ends = [dev([0], torch.int32), dev([0], torch.int32)]
    s.table.fill_(-1)
    n = [0] * B
    n_dev = s.counts(n)
    T = max(T0)
    k, v = randn(B, p.Hkv, T, p.D, seed=50), randn(B, p.Hkv, T, p.D, seed=51)
    new = dev(T0, torch.int32)
    lg.lg_paged_table_extend(p, n_dev, new, free, ends[0], s.table, ends[1])
    lg.lg_paged_append(p, *s.cache, s.table, k, v, n_dev, new)
    c.table = s.table.cpu().numpy()
    for b in range(B):
        c.append(b, 0, np64(k)[b, :, :T0[b]], np64(v)[b, :, :T0[b]])
    n = list(T0)
    k1, v1 = (torch.empty(B, p.Hkv, 1, p.D, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    q = torch.empty(B, p.Hq, p.D, dtype=torch.bfloat16, device="cuda")
    o, lse, ws = torch.empty_like(q), torch.empty(B, p.Hq, device="cuda"), lg.paged_decode_workspace(p)
    before, after = s.counts(n), s.counts(n)
    start, nxt = ends[1].clone(), dev([0], torch.int32)

    def step():
        after.copy_(before + 1)
        lg.lg_paged_table_extend(p, before, None, free, start, s.table, nxt, T_new=1)
        lg.lg_paged_append(p, *s.cache, s.table, k1, v1, before)
        lg.lg_paged_decode(p, q, *s.cache, s.table, after, o=o, lse=lse, workspace=ws)
        before.copy_(after)
        start.copy_(nxt)

    run = step
    if graph:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        run = g.replay
    for i in range(steps):
        k1.copy_(randn(*k1.shape, seed=200 + i)); v1.copy_(randn(*v1.shape, seed=300 + i)); q.copy_(randn(*q.shape, seed=400 + i))
        run()
        c.table = s.table.cpu().numpy()
        for b in range(B):
            c.append(b, n[b], np64(k1)[b], np64(v1)[b])
        n = [x + 1 for x in n]
        s.check_decode(q, o, lse, n)
    assert start.item() == sum(R.pages_of(x, c.sink, c.window, c.P) for x in n)
    s.same_state()
    assert lg.lg_last_status(ws) == 0
    return n


@pytest.mark.parametrize("graph", [False, True])
def test_serving_loop(lg, graph):
    _serve(lg, Setup(lg, [0] * 4, 8, 2, 128, 16, 80, 16, seed=4), 12, [1, 94, 200, 30], graph)


def test_serving_loop_d64_and_read_back(lg):
    """... then a chunk attends to what the loop left, and the cache is read back through its slot map."""
    s = Setup(lg, [0] * 3, 6, 2, 64, 64, 128, 32, seed=5)
    n = _serve(lg, s, 5, [10, 300, 1])
    T = max(n)
    slots = torch.empty(3, T, dtype=torch.int64, device="cuda")
    lg.lg_paged_slot_map(s.p, s.counts(n), s.counts([0] * 3), None, s.table, slots)
    k, v = lg.lg_paged_gather(s.p, *s.cache, slots)
    for b in range(3):
        for h in range(2):
            pos, ck, cv = s.ref.rows(b, h, n[b])
            for got, want in ((k, ck), (v, cv)):
                got = np64(got)[b, h]
                assert np.array_equal(got[pos], want)
                assert not np.delete(got, pos, axis=0).any()
    # one token as a chunk and as a step see the same keys, but for its own row, which the step reads in 8 bits
    q, k1, v1 = randn(3, 6, 1, 64, seed=7), randn(3, 2, 1, 64, seed=8), randn(3, 2, 1, 64, seed=9)
    full = dev(np.random.RandomState(2).permutation(s.num_pages)[:s.table.numel()].reshape(s.table.shape), torch.int32)
    table = torch.where(s.table >= 0, s.table, full)             # (pages for the step's token; any that nobody uses would do)
    o, _ = lg.lg_paged_chunk_prefill(s.p, q, k1, v1, *s.cache, s.table, n)
    exact = [torch.where(x == 0, x, torch.exp2(torch.floor(torch.log2(x.abs().float()))).to(x.dtype) * x.sign()) for x in (k1, v1)]
    o1, _ = lg.lg_paged_chunk_prefill(s.p, q, *exact, *s.cache, s.table, n)      # powers of two: exact in e4m3
    assert not torch.equal(o, o1)


def test_two_streams_with_a_workspace_each(lg):
    s = Setup(lg, [500, 900], 8, 2, 128, 64, 512, 32)
    qs = [randn(2, 8, 128, seed=i) for i in (1, 2)]
    want = [lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts()) for q in qs]
    n = s.counts()
    ws = [lg.paged_decode_workspace(s.p) for _ in qs]
    outs = [[torch.empty_like(q), torch.empty(2, 8, device="cuda")] for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    for _ in range(20):
        for q, w, (o, lse), st in zip(qs, ws, outs, streams):
            with torch.cuda.stream(st):
                lg.lg_paged_decode(s.p, q, *s.cache, s.table, n, o=o, lse=lse, workspace=w)
    torch.cuda.synchronize()
    for (o, lse), (wo, wl) in zip(outs, want):
        assert torch.equal(o, wo) and torch.equal(lse, wl)


def test_tensors_of_the_host_are_refused(lg):
    s = Setup(lg, [40], 2, 1, 64, 0, 64, 16)
    q, n = randn(1, 2, 64, seed=1), s.counts()
    for bad in ("q", "n", "table", "scale"):
        args = dict(q=q, n=n, table=s.table, scale=s.scales[0])
        args[bad] = args[bad].cpu()
        with pytest.raises(AssertionError):
            lg.lg_paged_decode(s.p, args["q"], *s.pools, args["scale"], s.scales[1], args["table"], args["n"], o=torch.empty_like(q))
    for wrong in (s.counts().int(), s.counts([1, 2])):
        with pytest.raises(AssertionError):
            lg.lg_paged_decode(s.p, q, *s.cache, s.table, wrong)
    k = randn(1, 1, 1, 64)
    with pytest.raises(lg.LgError):                               # one array for K and V
        lg.lg_paged_append(s.p, s.pools[0], s.pools[0], *s.scales, s.table, k, k, n)


def test_marshalled_calls(lg):
    s = Setup(lg, [40, 300], 8, 2, 128, 64, 256, 64)
    q, k, v = randn(2, 8, 128, seed=1), randn(2, 2, 1, 128, seed=2), randn(2, 2, 1, 128, seed=3)
    o, lse, ws = torch.empty_like(q), torch.empty(2, 8, device="cuda"), lg.paged_decode_workspace(s.p)
    append = lg.paged_append_call(s.p, *s.cache, s.table, k, v, s.counts())
    decode = lg.paged_decode_call(s.p, q, *s.cache, s.table, s.counts([41, 301]), o, lse, ws)
    append()
    decode()
    for b in range(2):
        s.ref.append(b, s.n[b], np64(k)[b], np64(v)[b])
    s.same_state()
    s.check_decode(q, o, lse, [41, 301])


@pytest.mark.parametrize("place", ["first", "last"])
@pytest.mark.parametrize("spread", [False, True])
@pytest.mark.parametrize("below", [24.6, 26.0])
def test_decode_many_small_weights_beside_a_large_one(lg, below, spread, place):
    """A token whose score is far above all others and whose V is zero, before or behind 131072 tokens of weights 2^-below that agree: what o holds is
    theirs alone.  A sequence for every warp, so that one warp works all of it; few pages, read again and again.  spread: one of the
    pages has a V scale 2^9 times the others'.

    Bound: as they stand relative to the large one, at 2^11, the weights are 2^-15 at least, where an f16 (steps of 2^-24) is off by up to 2^-10 of
    it; o is rounded to bf16 (2^-8); the fp32 sums of weights and of products run over n / 16 steps and the merges, (n / 16 + 64) 2^-23 each
    as everywhere here; 2^-14 for scores and exponentials.  What an f16 drops does not add up with n.  LSE: the sum's own error.
    """
    B, P, D, n = 1184, 128, 128, 131072
    p = lg.paged_params(B, 1, 1, D, 0, n + P, page_tokens=P, num_pages=4, scale=math.log(2.0) * below)
    k = torch.zeros(4, 1, P, D, device="cuda")
    v = torch.ones(4, 1, P, D, device="cuda")
    k[0, 0, 5, 0] = 1.0                                           # page 0: the large one at offset 5, alone or with others
    v[0, 0, 5] = 0.0
    v[2] = 2.0 ** -9                                              # page 2: under its larger scale the same as page 1
    table = torch.full((B, n // P + 1), 1, dtype=torch.int32, device="cuda")
    table[:, 0 if place == "first" else -1] = 0
    if spread:
        table[:, 600] = 2
    scale = torch.ones(4, 1, device="cuda")
    v_scale = scale.clone()
    v_scale[2] = 2.0 ** 9
    q = torch.zeros(B, 1, D, dtype=torch.bfloat16, device="cuda")
    q[:, 0, 0] = 1.0
    counts = torch.full((B,), n + P, dtype=torch.int64, device="cuda")
    o, lse = lg.lg_paged_decode(p, q, k.to(F8), v.to(F8), scale, v_scale, table, counts)
    tail = (n + P - 1) * 2.0 ** -below
    want = tail / (1 + tail)
    chain = (n / 16 + 64) * 2.0 ** -23
    assert np.abs(np64(o) - want).max() <= want * (2.0 ** -8 + 2.0 ** -10 + 2 * chain + 2.0 ** -14)
    assert np.abs(np64(lse) - (math.log(2.0) * below + math.log1p(tail))).max() <= chain + 2.0 ** -14


@pytest.mark.parametrize("n, T, sink", [([10, 100, 3, 400], 70, 64), ([90, 30], 16400, 0), ([3 + 100 * (b % 2) for b in range(140)], 70, 64)],
                         ids=["sinks", "long", "B140"])
@pytest.mark.parametrize("at", [0, -1])
def test_chunk_of_several_runs_with_an_absent_page_writes_nothing(lg, n, T, sink, at):
    """Sequences that are not worked together: a missing entry of the first or of the last leaves the others' results unwritten too."""
    B = len(n)
    s = Setup(lg, n, 1, 1, 64, sink, 64, 16)
    q, k, v = randn(B, 1, T, 64, seed=1), randn(B, 1, T, 64, seed=2), randn(B, 1, T, 64, seed=3)
    ws = lg.paged_chunk_prefill_workspace(s.p, T, n)
    clean = lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n, workspace=ws)
    assert lg.lg_last_status(ws) == 0
    _check_chunk_rows(s, n[:2], T, q, k, v, *clean, [0, T - 1], [0])
    good, s.ref.table = s.ref.table.copy(), s.ref.table.copy()
    s.ref.table[at, 0] = s.num_pages
    s.upload()
    o, lse = torch.full_like(q, 7.0), torch.full((B, 1, T), 7.0, device="cuda")
    lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n, o=o, lse=lse, workspace=ws)
    assert lg.lg_last_status(ws) == -7
    assert (o == 7).all() and (lse == 7).all()
    s.ref.table = good
    s.upload()
    lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n, o=o, lse=lse, workspace=ws)
    assert lg.lg_last_status(ws) == 0 and torch.equal(o, clean[0]) and torch.equal(lse, clean[1])


@pytest.mark.parametrize("D, window", [(128, 2048), (64, 2048), (128, 64)])
def test_chunk_row_that_is_nan(lg, D, window):
    """A NaN in one row of q is in that row's o and lse, and in no other's, whether the row's tile is cut along its keys (the long windows) or not."""
    n, T = [3000], 33
    s = Setup(lg, n, 2, 1, D, 128, window, 64)
    q, k, v = randn(1, 2, T, D, seed=1), randn(1, 1, T, D, seed=2), randn(1, 1, T, D, seed=3)
    clean = lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n)
    q[0, 1, 5, 7] = float("nan")
    o, lse = lg.lg_paged_chunk_prefill(s.p, q, k, v, *s.cache, s.table, n)
    assert torch.isnan(o[0, 1, 5]).all() and torch.isnan(lse[0, 1, 5])
    _check_chunk_rows(s, n, T, q, k, v, o, lse, [0, 4, 6, T - 1], [0, 1])
    assert torch.equal(o[0, 0], clean[0][0, 0]) and torch.equal(lse[0, 0], clean[1][0, 0])


def _check_averages(lg, bits, spread):
    """Scores of 2^bits, whose steps in fp32 are up to 2^11: o is an average of the V rows all the same, and the LSE that of the largest.

    A score is off by 2^-19 scale sum |q k|, as everywhere here, and its roundings on the way to a weight (2^-22 of it): `step`.  What is 2 steps and 30 below
    the largest has a weight below 2^-43; of the others any may have any weight.  o is rounded to bf16 (2^-8), weights to f16, which is not the sum's
    share (2^-11), and what f16 drops or the others weigh is below 2^-30 each, V as large as it may be."""
    n = [1024 - 7 * b for b in range(40)]
    s = Setup(lg, n, 4, 4, 64, 0, 1024, 32, scales=(-spread, spread))
    s.ref.scale[0][:] = 2.0 ** -7
    s.upload()
    q = (randn(40, 4, 64, seed=5).float() * 2.0 ** (bits - 1)).to(torch.bfloat16)
    o, lse = lg.lg_paged_decode(s.p, q, *s.cache, s.table, s.counts())
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    for b in (0, 1, 39):
        for h in range(4):
            pos, k, v = s.ref.rows(b, h, n[b])
            x = k @ np64(q[b, h]) / 8
            step = 2.0 ** -19 * (np.abs(k) @ np.abs(np64(q[b, h]))).max() / 8 + 2.0 ** -22 * np.abs(x).max()
            assert abs(lse[b, h].item() - x.max()) <= 2 * step + math.log(len(x)) + 2.0 ** -10
            near = v[x >= x.max() - 2 * step - 30]
            lo, hi = near.min(0), near.max(0)
            slack = (2.0 ** -8 + 2.0 ** -10) * np.maximum(np.abs(lo), np.abs(hi)) + len(x) * 2.0 ** -30 * np.abs(v).max(0)
            assert np.all(np64(o[b, h]) >= lo - slack) and np.all(np64(o[b, h]) <= hi + slack), (b, h)


@pytest.mark.parametrize("bits", [14, 20, 23, 24, 25, 26, 27, 28, 29, 30, 34])
def test_decode_scores_far_beyond_what_fp32_tells_apart(lg, bits):
    _check_averages(lg, bits, 0)


@pytest.mark.parametrize("bits", [6, 12, 18, 20, 24, 28, 34])
def test_decode_large_scores_over_scales_far_apart(lg, bits):
    """V scales that differ by up to 2^40 beside scores that fp32 holds in large steps: a scale weighs what it is, not what is left of it beside a score."""
    _check_averages(lg, bits, 20)
