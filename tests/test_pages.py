"""The paged dense cache on the GPU against 64 bits (tests/serving_ref.py derives the bounds)."""
import numpy as np
import pytest

from gpu_util import announce, lib_ready, torch_gpu
from serving_ref import attend, check, key_rows, rotate, rounding, torch_type, value_rows

pytestmark = pytest.mark.gpu


def pool(torch, kind, n_pages, H, page, d, layers=1, seed=0, fill=None):
    """Random pages; fill: a number everywhere instead."""
    g = torch.Generator().manual_seed(seed)
    shapes = ((layers, n_pages, H, page // 16, d // 8, 16, 8), (layers, n_pages, H, page // 8, d, 8))
    return [(torch.randn(s, generator=g) if fill is None else torch.full(s, fill)).to(torch_type(kind)).cuda() for s in shapes]


def deal(lens, page, columns=None, spare=2, seed=0):
    """A page table whose pages lie out of order, and the number of pages."""
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + spare
    order = np.random.default_rng(seed).permutation(n_pages)
    table, at = np.full((len(lens), columns or max(1, max(need))), -1, dtype=np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, n_pages


def i32(torch, x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


# ---- append ----------------------------------------------------------------------------------------

APPEND = [
    # new, held, Hq, Hkv, d, rot, interleaved, x, cache, page
    ([1], [0], 4, 1, 32, 32, False, "f32", "f16", 16),
    ([1, 1, 1, 1, 1], [0, 15, 16, 30, 400], 8, 2, 64, 64, False, "bf16", "bf16", 16),
    ([1, 1, 1], [7, 8, 31], 6, 3, 128, 64, True, "f16", "bf16", 32),
    ([16, 17, 15, 1], [0, 0, 0, 0], 4, 2, 64, 64, False, "f16", "f16", 16),
    ([9, 0, 40, 3], [7, 20, 9, 13], 4, 2, 96, 42, False, "bf16", "bf16", 32),
    ([130, 0, 0, 64, 257], [0, 0, 5, 61, 3], 2, 2, 128, 128, True, "f32", "bf16", 64),
    ([1000], [77], 16, 4, 128, 128, False, "bf16", "bf16", 256),
    ([33, 7], [1, 250], 0, 2, 256, 30, False, "f16", "f16", 128),     # keys alone
    ([20, 5], [3, 0], 4, 1, 160, 0, False, "f32", "f16", 16),         # nothing turns
    ([1001, 0, 1, 700, 700, 333], [5, 8, 0, 64, 3, 0], 3, 1, 64, 64, False, "bf16", "bf16", 32),   # two rows a workgroup, across sequences
    ([n % 4 for n in range(150)], [n % 23 for n in range(150)], 2, 1, 32, 32, True, "f16", "f16", 16),   # more than a wave's lanes
    ([1] * 70, list(range(70)), 2, 2, 64, 20, False, "bf16", "f16", 16),
    ([0] * 300 + [40] + [0] * 300 + [9, 1], [0] * 601 + [3, 7], 1, 1, 32, 32, False, "f32", "bf16", 16),
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: f"{len(c[0])}x{max(c[0])}-d{c[4]}-rot{c[5]}-{c[7]}-{c[8]}-p{c[9]}")
def test_append(case):
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache, RopeTable, rope_freqs
    new, held, Hq, H, d, rot, inter, tx, tc, page = case
    announce(f"append {case}")
    lens, N, B = [a + b for a, b in zip(new, held)], sum(new), len(new)
    table, n_pages = deal(lens, page)
    k, v = pool(torch, tc, n_pages, H, page, d, layers=2)
    k0, v0 = k.clone(), v.clone()
    g = torch.Generator().manual_seed(3)
    wide = torch.randn((N, (Hq + 2 * H) * d + 16), generator=g).to(torch_type(tx)).cuda()
    rows = wide[:, :(Hq + 2 * H) * d].unflatten(1, (Hq + 2 * H, d))
    q, kn, vn = (rows[:, :Hq] if Hq else None), rows[:, Hq:Hq + H], rows[:, Hq + H:]
    freq = rope_freqs(rot) if rot else None
    rope = RopeTable(freq, interleaved=inter, scale=1.5) if rot else None
    cache = PagedCache(k, v, i32(torch, table), i32(torch, lens), n_q_heads=max(Hq, H))
    cu = np.concatenate([[0], np.cumsum(new)])
    single = new == [1] * B
    q_out = cache.append(1, kn, vn, cu_new=None if single else i32(torch, cu), q=q, rope=rope)
    pos = np.concatenate([np.arange(n - m, n) for m, n in zip(new, lens)])
    turn = lambda x: rotate(x.double().cpu().numpy(), pos, freq.numpy(), inter, 1.5) if rot else (x.double().cpu().numpy(), 0.0)
    if Hq:
        want, tol = turn(q)
        check(q_out.double().cpu().numpy(), want, tol + rounding(np.abs(want) + tol, tc), "q")
    assert torch.equal(k[0], k0[0]) and torch.equal(v[0], v0[0])       # the other layer
    want, tol = turn(kn)
    tol = tol + rounding(np.abs(want) + tol, tc)
    K, K0 = key_rows(k[1].double().cpu().numpy()), key_rows(k0[1].double().cpu().numpy())
    V, V0 = value_rows(v[1].double().cpu().numpy()), value_rows(v0[1].double().cpu().numpy())
    plain = vn.float().to(torch_type(tc)).double().cpu().numpy()
    old = np.ones(K.shape[:1] + K.shape[2:3], bool)
    for r in range(N):
        b = int(np.searchsorted(cu, r, side="right")) - 1
        p, o = table[b, pos[r] // page], pos[r] % page
        check(K[p, :, o], want[r], tol[r] if rot else tol[r], f"key {r}")
        assert (V[p, :, o] == plain[r]).all(), f"value {r}"
        old[p, o] = False
    for x, x0 in ((K, K0), (V, V0)):
        assert (x == x0)[old[:, None, :, None].repeat(H, 1).repeat(d, 3)].all()    # every other token


def test_append_leaves_out_what_has_no_place():
    """Sequences of length 0 and shorter than their rows, pages that are none, rows past the table and behind
    the last start: nothing is stored, and the queries are turned all the same (those behind it are not)."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache, RopeTable, rope, rope_freqs
    announce("append without a place")
    page, H, d = 16, 2, 64
    table = np.array([[0, 1], [2, 3], [-1, 4], [5, 99], [6, 7]], dtype=np.int32)
    lens, new = [0, 2, 17, 33, 40], [1, 4, 2, 3, 10]                  # 40: past the table's 32
    k, v = pool(torch, "f16", 8, H, page, d)
    k0, v0 = k.clone(), v.clone()
    N = sum(new)
    cu = np.concatenate([[0], np.cumsum(new)])
    g = torch.Generator().manual_seed(3)
    rows = torch.randn((N + 3, 4 * H, d), generator=g).half().cuda()
    rope_t = RopeTable(rope_freqs(64))
    cache = PagedCache(k, v, i32(torch, table), i32(torch, lens), n_q_heads=2 * H)
    q_out = torch.full((N + 3, 2 * H, d), 5.0, dtype=torch.float16, device="cuda")
    cache.append(0, rows[:, 2 * H:3 * H], rows[:, 3 * H:], cu_new=i32(torch, cu), q=rows[:, :2 * H], rope=rope_t, q_out=q_out)
    pos = np.concatenate([np.arange(n - m, n) for m, n in zip(new, lens)])
    assert torch.equal(q_out[:N], rope(rows[:N, :2 * H], i32(torch, pos), rope_t))
    assert (q_out[N:] == 5.0).all()
    K, K0 = key_rows(k[0].cpu().numpy()), key_rows(k0[0].cpu().numpy())
    V, V0 = value_rows(v[0].cpu().numpy()), value_rows(v0[0].cpu().numpy())
    keys = rope(rows[:N, 2 * H:3 * H], i32(torch, pos), rope_t).cpu().numpy()
    stored = {}
    for r in range(N):
        b = int(np.searchsorted(cu, r, side="right")) - 1
        if 0 <= pos[r] < 32 and 0 <= table[b, pos[r] // page] < 8:
            stored[(int(table[b, pos[r] // page]), int(pos[r] % page))] = r
    assert len(stored) == 2 + 1 + 0 + 2                     # of sequences 1 to 4
    for p in range(8):
        for o in range(page):
            r = stored.get((p, o))
            assert (K[p, :, o] == (K0[p, :, o] if r is None else keys[r])).all(), (p, o)
            assert (V[p, :, o] == (V0[p, :, o] if r is None else rows[r, 3 * H:].cpu().numpy())).all(), (p, o)


@pytest.mark.parametrize("rot", [64, 42])
def test_append_turns_queries_in_place(rot):
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache, RopeTable, rope_freqs
    announce(f"append in place {rot}")
    lens = [40, 3, 17]
    table, n_pages = deal(lens, 16)
    cache = PagedCache(*pool(torch, "f16", n_pages, 2, 16, 64), i32(torch, table), i32(torch, lens), n_q_heads=6)
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn((24, h, 64), generator=g).half().cuda() for h in (6, 2, 2))
    cu, t = i32(torch, [0, 20, 20, 23]), RopeTable(rope_freqs(rot))
    want = cache.append(0, k, v, cu_new=cu, q=q, rope=t)
    want[23:] = q[23:]                                        # behind the last start
    assert cache.append(0, k, v, cu_new=cu, q=q, rope=t, q_out=q) is q
    assert torch.equal(q, want)


def test_append_at_given_positions():
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache, RopeTable, rope, rope_freqs
    announce("append at positions")
    table, n_pages = deal([5, 40], 16)
    k, v = pool(torch, "bf16", n_pages, 2, 16, 64)
    rows = torch.randn((2, 8, 64), device="cuda").bfloat16()
    pos, t = i32(torch, [1000000, -3]), RopeTable(rope_freqs(64))
    cache = PagedCache(k, v, i32(torch, table), i32(torch, [5, 40]), n_q_heads=4)
    q = cache.append(0, rows[:, 4:6], rows[:, 6:], q=rows[:, :4], rope=t, pos=pos)
    assert torch.equal(q, rope(rows[:, :4], pos, t))
    K = key_rows(k[0].float().cpu().numpy())
    want = rope(rows[:, 4:6], pos, t).float().cpu().numpy()
    assert (K[table[0, 0], :, 4] == want[0]).all() and (K[table[1, 2], :, 7] == want[1]).all()


# ---- decode ----------------------------------------------------------------------------------------

DECODE = [
    # lens, Hkv, G, d, page, type, window, pages taken out of (sequence, column)
    ([1], 1, 1, 32, 16, "f16", 0, []),
    ([0], 2, 4, 64, 16, "bf16", 0, []),
    ([0, 1, 15, 16, 17, 31, 32, 33], 2, 4, 64, 16, "f16", 0, []),
    ([5, 0, 47, 64, 65], 1, 3, 128, 16, "bf16", 0, []),
    ([48, 49, 130], 2, 16, 96, 32, "f16", 0, []),
    ([77, 300], 1, 17, 64, 64, "bf16", 0, []),               # groups of more than 16
    ([260], 2, 33, 32, 16, "f16", 0, []),
    ([1000], 2, 4, 128, 16, "f16", 0, []),
    ([1500, 3, 700], 3, 5, 160, 16, "bf16", 0, []),
    ([900, 0, 64], 1, 8, 192, 128, "f16", 0, []),
    ([500, 501], 2, 2, 224, 32, "bf16", 0, []),
    ([2100, 40], 2, 16, 256, 256, "bf16", 0, []),
    ([9000, 1], 1, 4, 128, 16, "f16", 0, []),
    ([100, 100, 33, 7], 2, 4, 64, 16, "f16", 33, []),
    ([100, 64, 1, 0], 2, 4, 128, 16, "bf16", 1, []),
    ([1024, 1000], 1, 7, 64, 16, "f16", 513, []),
    ([100, 40, 16], 2, 4, 64, 16, "bf16", 0, [(0, 0), (0, 3), (0, 6), (1, 1), (2, 0)]),
    ([600], 1, 4, 128, 16, "f16", 300, [(0, c) for c in range(20)] + [(0, 30)]),
    ([5000, 2000, 31], 2, 18, 64, 32, "bf16", 3001, [(0, c) for c in range(70)] + [(1, 9)]),
    ([1700] * 5 + [0, 1], 3, 4, 128, 16, "f16", 0, [(1, 50)]),
]


def decode_case(torch, case, seed=0, sharp=2.0, junk=float("nan"), spare=1):
    """spare: columns of the table past the longest sequence (many: a workgroup does not take a pair alone)."""
    lens, H, G, d, page, kind, window, gone = case
    table, n_pages = deal(lens, page, columns=-(-max(max(lens), 1) // page) + spare, seed=seed)
    rng = np.random.default_rng(seed)
    k, v = pool(torch, kind, n_pages, H, page, d, seed=seed)
    for b, c in gone:
        table[b, c] = rng.choice([-1, n_pages, 2 ** 31 - 1, -2 ** 31])
    # what no query sees holds junk
    seen = np.zeros((n_pages, page), bool)
    for b, n in enumerate(lens):
        for t in range(max(0, n - window) if window else 0, n):
            if 0 <= table[b, t // page] < n_pages:
                seen[table[b, t // page], t % page] = True
    mask = torch.from_numpy(~seen).cuda()
    k[0].view(n_pages, H, page // 16, d // 8, 16, 8).masked_fill_(mask.view(n_pages, 1, page // 16, 1, 16, 1), junk)
    v[0].view(n_pages, H, page // 8, d, 8).masked_fill_(mask.view(n_pages, 1, page // 8, 1, 8), junk)
    g = torch.Generator().manual_seed(seed + 1)
    q = (torch.randn((len(lens), H * G, d), generator=g) * sharp).to(torch_type(kind)).cuda()
    return table, k, v, q


def reference(case, table, k, v, q, sm_scale=None):
    K, V = (np.nan_to_num(f(x[0].double().cpu().numpy()), nan=0.0, posinf=0.0, neginf=0.0) for f, x in ((key_rows, k), (value_rows, v)))
    return attend(q.double().cpu().numpy(), K, V, table, case[0], case[6], sm_scale)


@pytest.mark.parametrize("spare", [1, 700])
@pytest.mark.parametrize("case", DECODE, ids=lambda c: f"{len(c[0])}x{max(c[0])}-h{c[1]}-g{c[2]}-d{c[3]}-p{c[4]}-{c[5]}-w{c[6]}-{len(c[7])}")
def test_decode(case, spare):
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce(f"page decode {case} {spare}")
    table, k, v, q = decode_case(torch, case, spare=spare)
    cache = PagedCache(k, v, i32(torch, table), i32(torch, case[0]), n_q_heads=q.shape[1])
    out = cache.decode(0, q, window=case[6])
    want, tol = reference(case, table, k, v, q)
    check(out.cpu().numpy(), want, tol, "decode")
    again = cache.decode(0, q, window=case[6], workspace=cache.workspace())
    assert torch.equal(out, again)                           # a fixed order: the same bits


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("junk", [float("inf"), float("-inf"), 60000.0])
def test_decode_sees_nothing_that_is_masked(kind, junk):
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce(f"page decode junk {kind} {junk}")
    case = ([1, 18, 100, 0], 2, 4, 64, 16, kind, 60, [(2, 4)])
    outs = []
    for j in (junk, 0.0):
        table, k, v, q = decode_case(torch, case, junk=j)
        outs.append(PagedCache(k, v, i32(torch, table), i32(torch, case[0]), n_q_heads=8).decode(0, q, window=60))
    assert torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_decode_of_extreme_scores(kind):
    """Peaked rows, whose scores lie hundreds apart, and flat ones; one number of the scale."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce(f"page decode extreme {kind}")
    case = ([700, 90], 2, 4, 128, 32, kind, 0, [])
    for sharp, sm in ((0.0, None), (60.0, None), (1.0, 3.0)):
        table, k, v, q = decode_case(torch, case, sharp=sharp)
        cache = PagedCache(k, v, i32(torch, table), i32(torch, case[0]), n_q_heads=8)
        want, tol = reference(case, table, k, v, q, sm)
        check(cache.decode(0, q, sm_scale=sm).cpu().numpy(), want, tol, f"sharp {sharp} sm {sm}")


def test_decode_rows_without_scores():
    """Scores of -inf alone give zeros; a NaN in a query is its row's alone."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce("page decode without scores")
    case = ([40, 20], 1, 4, 64, 16, "bf16", 0, [])
    table, k, v, q = decode_case(torch, case, junk=0.0)
    k[0, :, :, :, 0, :, 0] = float("inf")                    # channel 0 of every key
    q[:, :, 0] = -1.0
    cache = PagedCache(k, v, i32(torch, table), i32(torch, case[0]), n_q_heads=4)
    assert (cache.decode(0, q) == 0).all()
    table, k, v, q = decode_case(torch, case, junk=0.0)
    cache = PagedCache(k, v, i32(torch, table), i32(torch, case[0]), n_q_heads=4)
    want = cache.decode(0, q)
    q[0, 2, 5] = float("nan")
    out = cache.decode(0, q)
    assert torch.isnan(out[0, 2]).all()
    out[0, 2] = want[0, 2]
    assert torch.equal(out, want)


@pytest.mark.parametrize("B,top,H,G,d,spare", [(300, 40, 2, 2, 32, 1), (300, 40, 2, 2, 32, 300), (4096, 3, 2, 2, 32, 70), (70, 600, 2, 2, 32, 1),
                                               (70, 600, 2, 2, 32, 200), (4096, 2, 1, 16, 256, 70), (64, 1500, 8, 1, 32, 1), (65, 300, 1, 20, 64, 100)])
def test_decode_of_many_sequences(B, top, H, G, d, spare):
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce(f"page decode of {B} sequences")
    lens = np.random.default_rng(B).integers(0, top + 1, B).tolist()
    lens[-1] = top
    case = (lens, H, G, d, 16, "f16", 0, [])
    table, k, v, q = decode_case(torch, case, spare=spare)
    out = PagedCache(k, v, i32(torch, table), i32(torch, lens), n_q_heads=H * G).decode(0, q)
    want, tol = reference(case, table, k, v, q)
    check(out.cpu().numpy(), want, tol, "many")


@pytest.mark.parametrize("B,H", [(64, 8), (65, 8), (130, 4), (256, 2), (257, 2)])
def test_decode_longest_first(B, H):
    """A few long sequences among many short ones, of equal lengths some of them, in one launch."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce(f"page decode longest first {B} {H}")
    rng = np.random.default_rng(B)
    lens = np.where(rng.random(B) < 0.05, rng.integers(500, 768, B), rng.integers(0, 70, B))
    lens[B // 2] = lens[B - 1] = 768
    case = (lens.tolist(), H, 1, 256, 16, "f16", 0, [])
    table, k, v, q = decode_case(torch, case, spare=0)
    out = PagedCache(k, v, i32(torch, table), i32(torch, case[0]), n_q_heads=H).decode(0, q)
    want, tol = reference(case, table, k, v, q)
    check(out.cpu().numpy(), want, tol, "longest first")


def test_decode_lengths_and_queries_as_they_come():
    """Lengths below 0 and past the table are held to it; queries inside wider rows; the last of several layers."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce("page decode odd lengths")
    page, H, G, d = 16, 2, 4, 64
    k, v = pool(torch, "f16", 6, H, page, d, layers=3)
    table = np.array([[3, 1], [0, 5], [2, 4]], dtype=np.int32)
    wide = torch.randn((3, (H * G + 2 * H) * d), device="cuda").half()
    q = wide[:, :H * G * d].unflatten(1, (H * G, d))
    cache = PagedCache(k, v, i32(torch, table), i32(torch, [-7, 2 ** 31 - 1, 20]), n_q_heads=H * G)
    out = cache.decode(2, q)
    want, tol = attend(q.double().cpu().numpy(), key_rows(k[2].double().cpu().numpy()), value_rows(v[2].double().cpu().numpy()), table, [0, 32, 20])
    check(out.cpu().numpy(), want, tol, "odd lengths")


def test_pages_past_2_to_32():
    """Pages whose elements lie past 2^32: appended to and attended to."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce("pages past 2^32")
    H, page, d = 8, 256, 128
    n_pages = (1 << 32) // (H * page * d) + 3
    k = torch.zeros((1, n_pages, H, page // 16, d // 8, 16, 8), dtype=torch.float16, device="cuda")
    v = torch.zeros((1, n_pages, H, page // 8, d, 8), dtype=torch.float16, device="cuda")
    table = np.array([[n_pages - 1, 5, n_pages - 2]], dtype=np.int32)
    lens = i32(torch, [600])
    cache = PagedCache(k, v, i32(torch, table), lens, n_q_heads=16)
    rows = torch.randn((600, 2 * H, d), device="cuda").half()
    cache.append(0, rows[:, :H], rows[:, H:], cu_new=i32(torch, [0, 600]))
    q = torch.randn((1, 16, d), device="cuda").half()
    out = cache.decode(0, q)
    ids = torch.from_numpy(table[0].astype(np.int64)).cuda()
    K, V = key_rows(k[0, ids].double().cpu().numpy()), value_rows(v[0, ids].double().cpu().numpy())
    assert (K[0][:, :256] == rows[:256, :H].double().cpu().numpy().transpose(1, 0, 2)).all()
    assert (V[2][:, :88] == rows[512:, H:].double().cpu().numpy().transpose(1, 0, 2)).all()
    want, tol = attend(q.double().cpu().numpy(), K, V, np.array([[0, 1, 2]]), [600])
    check(out.cpu().numpy(), want, tol, "past 2^32")
    assert float(k[0, :5].abs().max()) == 0.0                # where a cut-off address would have landed


def test_decode_on_two_streams():
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce("page decode on two streams")
    case = ([3000, 50, 700], 2, 4, 128, 16, "bf16", 0, [])
    table, k, v, q = decode_case(torch, case)
    cache = PagedCache(k, v, i32(torch, table), i32(torch, case[0]), n_q_heads=8)
    want = cache.decode(0, q)
    qs = [q, (q * 0.5).to(q.dtype)]
    wants = [want, cache.decode(0, qs[1])]
    ws = [cache.workspace(), cache.workspace()]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(6):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                outs[i].append(cache.decode(0, qs[i], workspace=ws[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(o, wants[i]) for o in outs[i])


@pytest.mark.parametrize("G,d,columns", [(4, 64, 8), (4, 64, 100), (16, 256, 100)])
def test_step_captured(G, d, columns):
    """Append and decode in one graph that follows the lengths and the page table: replayed with the
    program's own work between, in a workspace that another graph shares."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache, RopeTable, rope_freqs
    announce(f"paged step captured {G} {d} {columns}")
    B, H, page = 3, 2, 16
    k, v = pool(torch, "f16", 24, H, page, d)
    table = torch.full((3, columns), -1, dtype=torch.int32, device="cuda")
    table[:, :8] = torch.arange(24, dtype=torch.int32, device="cuda").view(3, 8)[:, torch.randperm(8)]
    lens = i32(torch, [30, 0, 100])
    t = RopeTable(rope_freqs(64))
    cache = PagedCache(k, v, table, lens, n_q_heads=H * G)
    k2, v2 = k.clone(), v.clone()
    twin = PagedCache(k2, v2, table, lens, n_q_heads=H * G)
    rows = torch.randn((B, H * G + 2 * H, d), device="cuda").half()
    q_out, out, other = torch.empty((B, H * G, d), dtype=torch.float16, device="cuda"), torch.empty((B, H * G, d), device="cuda"), None
    ws = cache.workspace()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def step(c, o):
        qq = c.append(0, rows[:, H * G:H * G + H], rows[:, H * G + H:], q=rows[:, :H * G], rope=t, q_out=q_out)
        return c.decode(0, qq, out=o, workspace=ws)
    g, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    other = torch.empty_like(out)
    with torch.cuda.graph(g):
        step(cache, out)
    with torch.cuda.graph(g2):
        cache.decode(0, q_out, window=5, out=other, workspace=ws)
    for i in range(5):
        rows.normal_()
        lens += torch.tensor([1, 0 if i < 2 else 1, 1], dtype=torch.int32, device="cuda")
        if i == 3:
            table[2, 0] = -1                                  # a page given back
        g.replay()
        g2.replay()
        got, got2 = out.clone(), other.clone()
        torch.cuda.synchronize()
        q = twin.append(0, rows[:, H * G:H * G + H], rows[:, H * G + H:], q=rows[:, :H * G], rope=t)
        assert torch.equal(got, twin.decode(0, q)), i
        assert torch.equal(got2, twin.decode(0, q, window=5)), i
        assert torch.equal(k, k2) and torch.equal(v, v2)


# ---- numbers at the ends -----------------------------------------------------------------------------

def not_finite(v, case, table, want):
    """attend's results over the finite values alone, and in each channel that a sequence sees an infinity or a NaN
    in, what that makes of it: every finite score has a weight above 0."""
    lens, H, G, d, page, _, window, _ = case
    V, out = value_rows(v[0].double().cpu().numpy()), want.copy()
    for b, n in enumerate(lens):
        ts = [t for t in range(max(0, n - window) if window else 0, n) if 0 <= table[b, t // page] < V.shape[0]]
        for h in range(H):
            x = np.array([V[table[b, t // page], h, t % page] for t in ts]).reshape(-1, d)
            x = np.where(np.isfinite(x), 0.0, x)
            with np.errstate(invalid="ignore"):
                all_of = x.sum(0)
            out[b, h * G:(h + 1) * G] = np.where(all_of == 0, out[b, h * G:(h + 1) * G], all_of)
    return out


@pytest.mark.parametrize("case,spare", [
    (([1, 40, 700, 0], 2, 4, 64, 16, "f16", 0, []), 1),
    (([1, 40, 700, 0], 2, 4, 64, 16, "bf16", 0, []), 1),
    (([90, 3000, 33], 2, 4, 128, 16, "f16", 0, [(1, 40)]), 700),
    (([90, 3000, 33], 1, 16, 128, 32, "bf16", 0, []), 700),
    (([700, 2500], 1, 17, 64, 16, "f16", 600, []), 700),
    (([300, 65], 2, 3, 256, 16, "bf16", 0, []), 1),
    (([300, 2000], 1, 16, 256, 16, "f16", 0, []), 700),
    (([20] * 80, 2, 2, 32, 16, "bf16", 0, []), 700),
    (([200, 64, 70], 2, 4, 128, 16, "bf16", 90, [(0, 8)]), 1),
    (([130] * 40, 8, 1, 192, 64, "f16", 0, []), 0),
    (([4000, 90], 2, 5, 224, 16, "f16", 0, []), 700),
    (([1500], 1, 33, 160, 256, "bf16", 1200, []), 30),
], ids=lambda x: str(x) if isinstance(x, int) else f"{len(x[0])}x{max(x[0])}-g{x[2]}-d{x[3]}-{x[5]}")
@pytest.mark.parametrize("sharp", [2.0, 60.0])
def test_decode_of_infinite_values(case, spare, sharp):
    """An infinity that a sequence sees is its channel's output, however small its weight; both signs, or a NaN,
    make it NaN; other channels, heads and sequences are as they were.  Sharp: weights far below float32's range."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce(f"page decode of infinite values {case} {spare} {sharp}")
    table, k, v, q = decode_case(torch, case, spare=spare, sharp=sharp, junk=float("nan"))
    lens, H, page, window = case[0], case[1], case[4], case[6]
    rng = np.random.default_rng(4)
    put = []
    for b, n in enumerate(lens):
        if n == 0 or b % 3 == 2:
            continue
        first = max(0, n - window) if window else 0
        for c, signs in ((0, (1,)), (5, (-1,)), (17, (1, 1, 1)), (18, (1, -1)), (30, (0,)), (31, (1, 0))):
            for s in signs:
                t = int(rng.integers(first, n))
                put.append((table[b, t // page], int(rng.integers(H)), t % page, c, {1: np.inf, -1: -np.inf, 0: np.nan}[s]))
    for p, h, o, c, x in put:
        if 0 <= p < v.shape[1]:
            v[0, p, h, o // 8, c, o % 8] = x
    fin = v.clone()
    fin[~torch.isfinite(fin)] = 0
    want, tol = reference(case, table, k, fin, q)
    want = not_finite(v, case, table, want)
    assert not np.isfinite(want).all()
    out = PagedCache(k, v, i32(torch, table), i32(torch, lens), n_q_heads=q.shape[1]).decode(0, q, window=window)
    check(out.cpu().numpy(), want, tol, "infinite values")


@pytest.mark.parametrize("spare", [1, 700])
def test_decode_rows_without_scores_of_infinite_values(spare):
    """Scores of -inf alone give zeros whatever the values are."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce(f"page decode without scores, infinite values {spare}")
    case = ([40, 900], 1, 4, 64, 16, "bf16", 0, [])
    table, k, v, q = decode_case(torch, case, spare=spare, junk=0.0)
    k[0, :, :, :, 0, :, 0] = float("inf")                    # channel 0 of every key
    q[:, :, 0] = -1.0
    v[0, :, :, ::2, 3] = float("inf")
    v[0, :, :, ::3, 9] = float("nan")
    cache = PagedCache(k, v, i32(torch, table), i32(torch, case[0]), n_q_heads=4)
    assert (cache.decode(0, q) == 0).all()


@pytest.mark.parametrize("spare", [1, 700])
def test_decode_of_large_values(spare):
    """Values up to 2^112 / T are added up as others are; what the sums of larger ones make infinite keeps its
    sign, beside an infinity too, and changes no other channel."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce(f"page decode of large values {spare}")
    case = ([1, 500, 2000], 1, 4, 64, 16, "bf16", 0, [])
    table, k, v, q = decode_case(torch, case, spare=spare, junk=0.0)
    v[0, :, :, :, 3] *= 2.0 ** 98                            # 2^112 / 2000 is 2^101: normal numbers stay below 2^3
    plain = v.clone()
    v[0, :, :, :, 5] = 2.0 ** 127
    v[0, :, :, :, 6] = -2.0 ** 127
    v[0, table[1, 2], 0, 0, 7] = float("-inf")
    want, tol = reference(case, table, k, plain, q)
    out = PagedCache(k, v, i32(torch, table), i32(torch, case[0]), n_q_heads=4).decode(0, q).cpu().numpy()
    assert (out[:, :, 5] >= 2.0 ** 126).all() and (out[:, :, 6] <= -2.0 ** 126).all() and (out[1, :, 7] == -np.inf).all()
    out[:, :, 5:7], out[1, :, 7] = want[:, :, 5:7], want[1, :, 7]
    check(out, want, tol, "large values")


@pytest.mark.parametrize("spare", [1, 700])
def test_decode_of_the_lowest_scores(spare):
    """Finite scores near float32's lowest number have their softmax as others do: of the keys that score
    highest, all alike here, the mean of the values.  Weights are exact, l and the sums add up
    to T / 32 + 64 numbers, the values' products are exact: (T / 32 + 64) U and a division."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce(f"page decode of the lowest scores {spare}")
    case = ([70, 3000], 1, 2, 64, 16, "bf16", 0, [])
    table, k, v, q = decode_case(torch, case, spare=spare, junk=0.0)
    k[0], q[:] = 0.0, 0.0
    # times log2(e): -1.84e38, and -1.85e38 for every third token
    k[0, :, :, :, 0, :, 0] = 2.0 ** 63
    k[0, :, :, :, 0, ::3, 0] = 2.0 ** 63 * 1.0078125
    q[:, 0, 0] = -1.5 * 2.0 ** 63
    q[:, 1, 0] = 0.0                                          # and a row of even scores
    out = PagedCache(k, v, i32(torch, table), i32(torch, case[0]), n_q_heads=2).decode(0, q, sm_scale=1.0).cpu().numpy()
    V = value_rows(v[0].double().cpu().numpy())
    for b, n in enumerate(case[0]):
        x = np.array([V[table[b, t // 16], 0, t % 16] for t in range(n)])
        for r, of in ((0, [t for t in range(n) if t % 16 % 3]), (1, list(range(n)))):
            tol = (2 * (n / 32 + 64) + 2) * 2.0 ** -24 * np.abs(x[of]).mean(0)
            check(out[b, r], x[of].mean(0), tol, f"lowest scores {b} {r}")


def test_decode_window_without_end():
    """The largest window is none: the same kernels, so the same bits."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce("page decode window without end")
    for case, spare in ((([20000, 700], 1, 4, 128, 16, "bf16", 0, []), 1), (([600, 5], 2, 4, 128, 16, "f16", 0, []), 1),
                        (([300] * 40, 8, 1, 128, 16, "f16", 0, []), 400)):
        table, k, v, q = decode_case(torch, case, spare=spare)
        cache = PagedCache(k, v, i32(torch, table), i32(torch, case[0]), n_q_heads=q.shape[1])
        for window in (2 ** 31 - 1, 2 ** 31 - 31, 2 ** 31 - 30, 2 ** 30):
            assert torch.equal(cache.decode(0, q, window=window), cache.decode(0, q)), (case, window)


def test_decode_on_two_streams_without_workspaces():
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce("page decode on two streams without workspaces")
    case = ([3000, 50, 700], 2, 4, 128, 16, "bf16", 0, [])
    table, k, v, q = decode_case(torch, case)
    cache = PagedCache(k, v, i32(torch, table), i32(torch, case[0]), n_q_heads=8)
    args = [(q, 0), ((q * 0.5).to(q.dtype), 40)]                # another window: another plan
    wants = [cache.decode(0, x, window=w) for x, w in args]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(6):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                outs[i].append(cache.decode(0, args[i][0], window=args[i][1]))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(o, wants[i]) for o in outs[i])


def test_decode_captured_without_a_workspace():
    """Two graphs with workspaces of their own, replayed with eager calls between them."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache
    announce("page decode captured without a workspace")
    case = ([3000, 50, 700], 2, 4, 128, 16, "f16", 0, [])
    table, k, v, q = decode_case(torch, case)
    lens = i32(torch, case[0])
    cache = PagedCache(k, v, i32(torch, table), lens, n_q_heads=8)
    outs, graphs = [torch.empty(cache.shape, device="cuda") for _ in range(2)], []
    for o, window in zip(outs, (0, 100)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            cache.decode(0, q, window=window, out=o)
    for i in range(4):
        lens -= 1
        for g in graphs:
            g.replay()
        got = [o.clone() for o in outs]
        torch.cuda.synchronize()
        for o, window in zip(got, (0, 100)):
            assert torch.equal(o, cache.decode(0, q, window=window)), i
