"""One decode workspace, zero-filled once, serves calls of any size in turn: each result is that of a workspace of its own."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def lg():
    from paper_2410_01485_b200 import binding, build
    build.build()
    binding.load_library()
    return binding


def randn(*shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


def paged(lg, B, Hq, Hkv, D, window, n, P=64):
    cols = -(-window // P)
    p = lg.paged_params(B, Hq, Hkv, D, 0, window, page_tokens=P, num_pages=B * cols)
    pools = [(randn(B * cols, Hkv, P, D, seed=s) * 100).to(F8) for s in (1, 2)]
    scales = [torch.full((B * cols, Hkv), 2.0 ** -7, device="cuda") for _ in "kv"]
    table = torch.arange(B * cols, dtype=torch.int32, device="cuda").flip(0).view(B, cols)
    q, counts = randn(B, Hq, D, seed=3).bfloat16(), torch.tensor(n, dtype=torch.int64, device="cuda")
    return p, lambda o, lse, ws: lg.lg_paged_decode(p, q, *pools, *scales, table, counts, o=o, lse=lse, workspace=ws)


def check_in_turn(lg, make, calls, new_workspace):
    calls = [make(lg, *c) for c in calls]
    sizes = [new_workspace(p).numel() for p, _ in calls]
    shared = torch.zeros(max(sizes), dtype=torch.uint8, device="cuda")
    for p, run in calls:
        got = [torch.full((p.B, p.Hq, p.D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((p.B, p.Hq), 7.0, device="cuda")]
        want = [x.clone() for x in got]
        run(*got, shared)
        run(*want, new_workspace(p))
        for g, w in zip(got, want):
            bits = torch.int16 if g.dtype == torch.bfloat16 else torch.int32       # (some codes are NaN, and so are what attends them)
            assert torch.equal(g.view(bits), w.view(bits)), (p.B, p.Hq, p.Hkv, p.D)
    assert lg.lg_last_status(shared) == 0


def test_paged_decode(lg):
    uneven = [2048 - 300 * b if b != 5 else 1 for b in range(7)]
    check_in_turn(lg, paged, [
        (1, 64, 8, 128, 2048, [2048]), (9, 64, 8, 128, 2048, [2048] * 9), (8, 64, 8, 128, 2048, [5000] * 8), (16, 64, 8, 128, 2048, [2048] * 16),
        (9, 64, 8, 128, 2048, [2048 - b for b in range(9)]), (7, 16, 2, 64, 2048, uneven), (1, 16, 2, 64, 2048, [2000]), (40, 64, 8, 64, 2048, [2048] * 40),
        (7, 16, 2, 64, 2048, uneven), (50, 64, 8, 128, 640, [640] * 50), (3, 24, 2, 128, 2048, [2048, 700, 1]), (9, 64, 8, 128, 2048, [2048] * 9),
    ], lg.paged_decode_workspace)


def ring(lg, B, Hq, Hkv, D, window, n):
    p = lg.decode_params(B, Hq, Hkv, D, 0, window)
    k, v = (randn(B, Hkv, window, D, seed=s).bfloat16() for s in (1, 2))
    q, counts = randn(B, Hq, D, seed=3).bfloat16(), torch.tensor(n, dtype=torch.int64, device="cuda")
    return p, lambda o, lse, ws: lg.lg_sparse_decode(p, q, k, v, counts, o=o, lse=lse, workspace=ws)


# rings of 2048 tokens; (B, Hq, Hkv, D, window, n): few sequences, more of them, other head counts and dimensions, many units, and
# (2100 sequences) the schedule that needs no counters
RINGS = [
    (1, 64, 8, 128, 2048, [2048]), (9, 64, 8, 128, 2048, [2048] * 9), (8, 64, 8, 128, 2048, [5000] * 8), (16, 64, 8, 128, 2048, [2048] * 16),
    (2100, 1, 1, 64, 32, [20] * 2100), (9, 64, 8, 128, 2048, [2048 - b for b in range(9)]), (7, 16, 2, 64, 2048, [2048, 1, 0, 700, 2000, 64, 17]),
    (1, 16, 2, 64, 2048, [2000]), (40, 64, 8, 64, 2048, [2048] * 40), (50, 64, 8, 128, 640, [640] * 50), (9, 64, 8, 128, 2048, [2048] * 9),
]


def test_ring_decode(lg):
    check_in_turn(lg, ring, RINGS, lg.decode_workspace)


def test_decode_of_the_fixed_array(lg):
    """The same in turn over the array of the library, which every call of the process shares."""
    for c in RINGS:
        p, run = ring(lg, *c)
        if lg.decode_workspace(p).numel() > lg.DECODE_STATIC_SCRATCH_BYTES:
            continue
        q, k, v = randn(p.B, p.Hq, p.D, seed=3).bfloat16(), *(randn(p.B, p.Hkv, c[4], p.D, seed=s).bfloat16() for s in (1, 2))
        n = torch.tensor(c[5], dtype=torch.int64, device="cuda")
        o, lse = torch.full_like(q, 7.0), torch.full((p.B, p.Hq), 7.0, device="cuda")
        want, want_lse = torch.empty_like(o), torch.empty_like(lse)
        lg.lg_sparse_decode_static(p, q, k, v, n, o, lse)
        run(want, want_lse, lg.decode_workspace(p))
        assert torch.equal(o, want) and torch.equal(lse, want_lse), c[:5]


def test_both_caches(lg):
    """Calls over the ring and over pages on one workspace."""
    check_in_turn(lg, lambda lg, make, *c: make(lg, *c), [
        (ring, 1, 64, 8, 128, 2048, [2048]), (paged, 9, 64, 8, 128, 2048, [2048] * 9), (paged, 1, 64, 8, 128, 2048, [2048]),
        (ring, 9, 64, 8, 128, 2048, [2048] * 9), (paged, 40, 64, 8, 64, 1024, [1024] * 40), (ring, 40, 64, 8, 64, 1024, [1024] * 40),
    ], lambda p: lg.paged_decode_workspace(p) if isinstance(p, lg.PagedParams) else lg.decode_workspace(p))
