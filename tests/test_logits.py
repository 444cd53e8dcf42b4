"""Rows of logits made into probabilities on the GPU against 64 bits (tests/serving_ref.py derives the bounds)."""
import numpy as np
import pytest

from gpu_util import announce, lib_ready, torch_gpu
from serving_ref import check, rounding, shape_logits, torch_type

pytestmark = pytest.mark.gpu

CASES = [
    # rows, vocab, history, in, out, probs, rules
    (1, 1, 3, "f32", "f32", True, "ph"),
    (1, 7, 0, "f16", "f32", True, "p"),
    (2, 33, 5, "bf16", "bf16", True, "phm"),
    (3, 1000, 50, "f32", "f32", False, "phbm"),
    (3, 1001, 700, "f16", "f16", False, "phb"),
    (5, 4097, 3000, "bf16", "f32", True, "phbm"),
    (4, 12289, 100, "f32", "f16", True, "hbm"),
    (2, 40000, 9000, "f32", "f32", True, "phbm"),
    (70, 66000, 40, "bf16", "bf16", True, "phbm"),         # the longer runs
    (300, 20000, 64, "f16", "f32", True, "ph"),
    (70, 66000, 40, "f16", "f32", True, "phb"),
    (128, 66000, 300, "bf16", "f32", True, "phbm"),          # the longest, whose second launch counts again
    (110, 78001, 17000, "f32", "f32", True, "ph"),           # or does not
    (128, 66003, 100, "f32", "bf16", True, "b"),
    (300, 16500, 90, "f32", "f32", True, "pbm"),            # 128 KB of counts
    (6, 500, 30, "f32", "f32", True, ""),
    (6, 500, 30, "f32", "bf16", False, "m"),
]


def make(torch, rows, V, L, kind, rules, S=None, seed=0, gap=0):
    rng = np.random.default_rng(seed)
    S = rows if S is None else S
    wide = torch.from_numpy(rng.normal(0, 3, (rows, V + gap))).to(torch_type(kind)).cuda()
    arg = {}
    if "p" in rules:
        arg["params"] = np.stack([rng.uniform(0.7, 1.5, S), rng.uniform(-0.3, 1, S), rng.uniform(-0.2, 0.6, S), rng.uniform(0.5, 1.5, S)], 1).astype(np.float32)
    if "h" in rules:
        h = (rng.random((S, L)) ** 3 * V).astype(np.int32)
        h[rng.random((S, L)) < 0.05] = -1                  # ids that are no tokens
        h[rng.random((S, L)) < 0.02] = V
        arg["history"] = h
        arg["history_len"] = rng.integers(0, L + 1, S).astype(np.int32)
        arg["history_len"][0] = L + 5                       # held to the row
        arg["prompt_len"] = (arg["history_len"] * rng.random(S)).astype(np.int32)
    if "b" in rules:
        n = rng.integers(0, 40, S)
        n[0] = 700                                          # more than a workgroup's threads
        cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        ids = rng.integers(0, V, cu[-1]).astype(np.int32)
        ids[::7] = ids[0]                                   # one listed often
        ids[3::11] = -4
        ids[5::13] = V + 2
        arg["bias"] = (cu, ids, rng.normal(0, 2, cu[-1]).astype(np.float32))
    if "m" in rules:
        m = rng.integers(0, 2 ** 32, (rows, (V + 31) // 32 + 1), dtype=np.uint64).astype(np.uint32)
        m[rows // 2] = 0                                    # a row that allows nothing
        arg["mask"] = m.view(np.int32)
    return wide[:, :V], arg


def on_gpu(torch, arg):
    up = lambda x: tuple(up(y) for y in x) if isinstance(x, tuple) else torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return {k: up(v) for k, v in arg.items()}


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c))
def test_logits(case):
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import LogitsRules, adjust_logits
    rows, V, L, ti, to, probs, rules = case
    announce(f"logits {case}")
    l, arg = make(torch, rows, V, L, ti, rules, gap=(0, 3, 8)[rows % 3])
    out = torch.full((rows, V), 9.0, dtype=torch_type(to), device="cuda")
    assert adjust_logits(l, LogitsRules(**on_gpu(torch, arg)), probs=probs, out=out) is out
    want, tol = shape_logits(l.double().cpu().numpy(), probs=probs, **arg)
    fin = np.where(np.isfinite(want), np.abs(want), 0.0) + tol
    check(out.double().cpu().numpy(), want, tol + rounding(fin, to), "logits")


@pytest.mark.parametrize("probs", [False, True])
@pytest.mark.parametrize("V", [50, 5000])
def test_logits_of_trees(V, probs):
    """Paths behind the histories of their sequences: a chain of 64, a bushy tree, none, one node, absent nodes."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree, LogitsRules, adjust_logits
    announce(f"logits of trees {V}")
    rng = np.random.default_rng(V)
    trees = [list(range(-1, 63)), [-1] + [int(rng.integers(i)) for i in range(1, 40)], [], [-1], [-1, 0, -2, 5, 1, 2]]
    cu = np.concatenate([[0], np.cumsum([len(t) for t in trees])]).astype(np.int32)
    parent, N = np.array(sum(trees, []), dtype=np.int32), int(cu[-1])
    token = rng.integers(-1, V + 1, N).astype(np.int32)
    l, arg = make(torch, N, V, 200, "f32", "phbm", S=len(trees))
    tree = DraftTree(cu, torch.from_numpy(parent).cuda())
    out = adjust_logits(l, LogitsRules(**on_gpu(torch, arg)), tree=tree, token=torch.from_numpy(token).cuda(), probs=probs)
    want, tol = shape_logits(l.double().cpu().numpy(), probs=probs, tree=(cu, parent), token=token, **arg)
    check(out.cpu().numpy(), want, tol, "trees")


def test_greedy_rows():
    """Temperature 0: one at the first largest, ties to the lowest index, across runs; nothing where nothing is allowed."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import LogitsRules, adjust_logits
    announce("greedy rows")
    V = 20000
    l = torch.zeros((7, V), device="cuda")
    l[0, [19999, 4095, 8192]] = 2.0
    l[1] = -5.0
    l[2] = float("-inf")
    l[3] = float("-inf")
    l[3, 12345] = -3e38
    l[4, 17] = float("nan")
    l[4, [18, 9000]] = 1.0
    l[5, 7000] = float("inf")
    l[6, 0] = float("nan")
    params = torch.tensor([[1.0, 0.0, 0.0, t] for t in (0.0, -1.0, 0.0, 0.0, 0.0, float("nan"), 0.0)], device="cuda")
    out = adjust_logits(l, LogitsRules(params=params))
    want = torch.zeros_like(out)
    for r, i in ((0, 4095), (1, 0), (3, 12345), (4, 18), (5, 7000), (6, 1)):
        want[r, i] = 1.0
    assert torch.equal(out, want)


@pytest.mark.parametrize("V", [900, 30000])
def test_temperatures_at_the_ends(V):
    """+inf makes what is allowed even; the smallest ones, whose inverse is no float32, leave the largest entries."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import LogitsRules, adjust_logits
    announce(f"temperatures at the ends {V}")
    l = torch.randn((3, V), generator=torch.Generator().manual_seed(1)).cuda()
    l[:, [5, V - 1]] = 9.0
    l[:, 7] = float("-inf")
    params = torch.tensor([[1.0, 0.0, 0.0, t] for t in (float("inf"), 1e-38, 1e-45)], device="cuda")
    out = adjust_logits(l, LogitsRules(params=params)).double()
    even = torch.full((V,), 1 / (V - 1), dtype=torch.float64, device="cuda")
    even[7] = 0
    # a sum of V ones is exact, its inverse and the product rounded
    assert ((out[0] - even).abs() <= 2 ** -22 * even).all()
    assert (out[1:, [5, V - 1]] == 0.5).all() and (out[1:].sum(1) == 1).all()


def test_rows_that_are_not_numbers():
    """Masked NaN and infinities count for nothing; one that is not masked makes its row NaN and no other."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import LogitsRules, adjust_logits
    announce("logits that are not numbers")
    V = 9000
    l = torch.randn((4, V), device="cuda")
    bad = torch.zeros(V, dtype=torch.bool, device="cuda")
    bad[[5, 4100, 8999]] = True
    word = torch.zeros(-(-V // 32) * 32, dtype=torch.int64, device="cuda")
    word[:V] = (~bad).long()
    word = (word.view(-1, 32) << torch.arange(32, device="cuda")).sum(1)
    mask = torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32).repeat(4, 1)
    clean = adjust_logits(l, LogitsRules(mask=mask))
    l[0, 5], l[1, 4100], l[2, 8999] = float("nan"), float("inf"), float("-inf")
    assert torch.equal(adjust_logits(l, LogitsRules(mask=mask)), clean)
    out = adjust_logits(l, LogitsRules())
    assert torch.isnan(out[0]).all() and torch.isnan(out[1]).all() and out[2, 8999] == 0
    assert torch.equal(out[3], adjust_logits(l[3:], LogitsRules())[0])
    low = torch.full((2, V), torch.finfo(torch.float32).min, device="cuda")       # a mask of the type's lowest value
    low[1, 6000] = 0.0
    out = adjust_logits(low, LogitsRules())
    assert (out[0] - 1 / V).abs().max() <= 2 ** -20 / V and out[1, 6000] == 1 and out[1].sum() == 1


@pytest.mark.parametrize("kind,probs", [("f32", True), ("f32", False), ("bf16", True), ("f16", False)])
def test_logits_in_place(kind, probs):
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import LogitsRules, adjust_logits
    announce(f"logits in place {kind} {probs}")
    l, arg = make(torch, 5, 9001, 60, kind, "phb")
    l = l.contiguous()
    rules = LogitsRules(**on_gpu(torch, arg))
    want = adjust_logits(l, rules, probs=probs, out=torch.empty_like(l))
    assert adjust_logits(l, rules, probs=probs, out=l) is l
    assert torch.equal(l, want)


def test_logits_captured():
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import LogitsRules, adjust_logits, adjust_logits_workspace
    announce("logits captured")
    l, arg = make(torch, 3, 10000, 200, "f32", "phbm")
    l = l.contiguous()
    a = on_gpu(torch, arg)
    a["history_len"].fill_(50)
    rules, out, ws = LogitsRules(**a), torch.empty((3, 10000), device="cuda"), adjust_logits_workspace(l)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        adjust_logits(l, rules, out=out, workspace=ws)
    for i in range(4):
        a["history_len"] += 10
        l.mul_(0.9)
        g.replay()
        got = out.clone()
        torch.cuda.synchronize()
        assert torch.equal(got, adjust_logits(l, rules)), i


@pytest.mark.parametrize("V", [900, 30000])
def test_temperatures_over_the_whole_range(V):
    """Rows that hold float32's lowest and highest numbers, at temperatures as large: +inf makes them even too.
    There an exponent is at most 2^128 halved, times twice the smallest number, 2^-149: off by 2^-21, and
    the sum as much."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import LogitsRules, adjust_logits
    announce(f"temperatures over the whole range {V}")
    temps = [float("inf"), 3.4e38, 3e38, 1e38, 1.2e38, 2e37, 1e30]
    big = torch.finfo(torch.float32).max
    l = torch.randn((len(temps), V), generator=torch.Generator().manual_seed(2)).cuda()
    l[:, ::5] = -big
    l[:, 3::7] = big
    l[:, 6::11] = big / 3
    l[:, 8] = float("-inf")
    params = torch.tensor([[1.0, 0.0, 0.0, t] for t in temps], dtype=torch.float32, device="cuda")
    out = adjust_logits(l, LogitsRules(params=params)).cpu().numpy()
    host, par = l.double().cpu().numpy(), params.cpu().numpy()
    want, tol = shape_logits(host[1:], par[1:], probs=True)
    even = np.full((1, V), 1 / (V - 1))
    even[0, 8] = 0
    check(out[:1], even, 2.0 ** -20 * even, "temperature inf")
    check(out[1:], want, tol, "large temperatures")
