"""What a row of dwkv_tree_decode keeps beside rows, tokens and scales of quite
another size, against plain float64 attention.  Tolerances are those of
test_tree_decode (its `bound`), from the scores of the rows compared, unless a
test derives its own."""
import numpy as np
import pytest

from gpu_util import announce, device_cache, lib_ready, torch_gpu
import test_tree_decode
from oracle.factorized import reconstruct
from test_tree_decode import D, bound, check, inputs, make_host, make_tree, reference

pytestmark = pytest.mark.gpu


def run(host, cu, parent, q, k, v, layer=0, split=0, sm_scale=None):
    torch = torch_gpu()
    from paper_2607_06523_amd import DraftTree
    tree = DraftTree(cu, torch.from_numpy(np.asarray(parent, dtype=np.int32)).cuda())
    return device_cache(host, split_tokens=split).tree_decode(layer, tree, q.cuda(), k.cuda(), v.cuda(), sm_scale=sm_scale).cpu().numpy()


@pytest.mark.parametrize("fmt,rb", [("f16", 48), ("int8", 32), ("f16", 96)])
@pytest.mark.parametrize("power", [20, 30, 40, 100])
def test_rows_beside_large_queries(power, fmt, rb):
    """Ordinary nodes and heads share blocks of 32 rows with bf16 queries 2^power times as large.  The ordinary rows keep
    the bound of their own scores.  The large rows' softmax is one-hot: what is left is a value's own error, 2^-21."""
    torch_gpu()
    lib_ready()
    host = make_host([600], 4, rb, fmt=fmt)
    rng = np.random.default_rng(21)
    cu, parent = make_tree([9], "tree", rng)
    q, k, v = inputs(host, 9, rng)
    big = np.zeros((9, 8), bool)
    big[3:5] = True                                     # whole nodes
    big[6:, 1::4] = True                                # one head of a group
    q[big] *= 2.0 ** power
    announce(f"tree decode rows beside queries of 2^{power} {fmt} {rb}")
    got = run(host, cu, parent, q, k, v)
    want, _ = reference(host, 0, cu, parent, q.double().numpy(), k.double().numpy(), v.double().numpy())
    small = q.clone()
    small[big] = 0.0
    _, top = reference(host, 0, cu, parent, small.double().numpy(), k.double().numpy(), v.double().numpy())
    check(got[~big], want[~big], bound(host, top), f"ordinary rows, 2^{power}")
    check(got[big], want[big], 2.0 ** -21 * 4, f"large rows, 2^{power}")


def test_large_queries_of_other_nodes_change_nothing():
    """Large finite numbers in a sibling's query, in an absent node's and in its child's: the other rows are equal bit by
    bit."""
    torch = torch_gpu()
    lib_ready()
    host = make_host([333, 70], 4, 48, seed=9)
    rng = np.random.default_rng(4)
    cu = np.array([0, 8, 13], dtype=np.int32)
    parent = np.array([-1, 0, 0, 1, -2, 4, 4, 2] + [-1, 0, 9, 2, 0], dtype=np.int32)
    q, k, v = inputs(host, 13, rng)
    want = run(host, cu, parent, q, k, v)
    other = [3, 4, 5, 6, 10, 11]                        # a leaf, absent nodes and nodes below them
    rest = [i for i in range(13) if i not in other]
    for fill in (1e30, -3e38, 1e12, float("inf"), float("nan")):
        q2 = q.clone()
        q2[other] = fill
        announce(f"tree decode, other nodes' queries {fill}")
        got = run(host, cu, parent, q2, k, v)
        assert np.array_equal(got[rest], want[rest]), fill
        assert np.all(got[[4, 5, 6, 10, 11]] == 0), fill


@pytest.mark.parametrize("fmt", ["f16", "int8"])
@pytest.mark.parametrize("small", ["queries", "sm_scale", "basis rows"])
@pytest.mark.parametrize("shift", [8, 13])
def test_small_projections_of_large_coefficients(shift, small, fmt):
    """Coefficients 2^shift times as large and queries, sm_scale or some rows of the bases so much smaller: the scores stay
    and so does their bound."""
    torch_gpu()
    lib_ready()
    host = make_host([800, 90], 4, 48, fmt=fmt)
    rng = np.random.default_rng(33)
    cu, parent = make_tree([9, 5], "tree", rng)
    q, k, v = inputs(host, 14, rng)
    f = 2.0 ** shift
    rows = slice(16, 32) if small == "basis rows" else slice(0, 48)
    if fmt == "int8":
        host.coef_scale_k[:, :, rows.start // 16:rows.stop // 16] *= np.float16(f)
    else:
        host.coef_k[..., rows] *= np.float16(f)
    scale = D ** -0.5
    if small == "basis rows":
        host.basis[:, :, :, 0, rows] /= np.float16(f)
    else:
        host.res_scale[:, 0] *= np.float16(f)
        if small == "queries":
            q /= f
        else:
            scale /= f
    announce(f"tree decode small {small} 2^-{shift} {fmt}")
    got = run(host, cu, parent, q, k, v, layer=1, sm_scale=scale)
    want, top = reference(host, 1, cu, parent, q.double().numpy(), k.double().numpy(), v.double().numpy(), scale=scale)
    assert 0.5 < top < 20.0
    check(got, want, bound(host, top), f"small {small} 2^-{shift} {fmt}")


@pytest.mark.parametrize("fmt", ["f16", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_scores_of_minus_infinity_leave_the_rest(monkeypatch, dtype, fmt):
    """The first 400 tokens of a sequence have infinite key scales, which stay with their entries and make their every
    score -inf; the other tokens' scores and the drafted keys' lie far below zero.  The rows are the attention of what is
    not -inf, in a sequence of such tokens alone that of the nodes."""
    torch_gpu()
    lib_ready()
    host = make_host([1000, 90], 4, 32, (2,), fmt=fmt, dtype=dtype)
    rng = np.random.default_rng(17)
    host.res_val[:, 0] = 0xFF                           # every key code -1
    host.res_scale[:, 0] = np.float16(4000.0)
    off = np.zeros(1090, bool)
    off[:400] = off[1000:] = True
    cu, parent = make_tree([10, 4], "tree", rng)
    q, k, v = inputs(host, 14, rng)
    q = q.abs() + 0.25
    k[:10] = -60.0
    finite = reconstruct

    def with_infinite_scales(h, layer, z, head, b):
        X = finite(h, layer, z, head, b)
        if z == 0:                                      # from the finite scales' keys
            t0, t1 = int(host.cu_seqlens[b]), int(host.cu_seqlens[b + 1])
            for t in np.nonzero(off[t0:t1])[0]:
                e = int(host.res_off[layer // host.window, head, t0 + t])
                X[t, host.res_idx[layer, 0, head, e:e + 2]] = -np.inf
        return X
    monkeypatch.setattr(test_tree_decode, "reconstruct", with_infinite_scales)
    want, _ = reference(host, 0, cu, parent, q.double().numpy(), k.double().numpy(), v.double().numpy())
    K = finite(host, 0, 0, 0, 0)[400:]
    top = max(float(np.abs(K @ q[i, h].double().numpy()).max()) for i in range(10) for h in range(4)) * D ** -0.5 * 1.4427
    assert np.all(np.isfinite(want)) and 300.0 < top < 6000.0
    host.res_scale[:, 0, :, off] = np.inf
    announce(f"tree decode, scores of -inf {fmt} {dtype}")
    got = run(host, cu, parent, q, k, v, split=1024)
    check(got, want, bound(host, top), f"scores of -inf {fmt} {dtype}")


@pytest.mark.parametrize("fmt,rb", [("f16", 48), ("int8", 32), ("f16", 112)])
@pytest.mark.parametrize("place", [3, 500, 890])
def test_large_value_scale_of_a_token_not_attended_to(place, fmt, rb):
    """One token's value scale is 2^25 times the others', which are all that most rows attend to (its probability is below
    2^-50 there); the values are residuals alone.  Two nodes attend to that token instead."""
    torch = torch_gpu()
    lib_ready()
    host = make_host([900, 70], 4, rb, (4, 16), fmt=fmt)
    rng = np.random.default_rng(place)
    host.coef_v[...] = 0
    host.res_scale[:, 1] = (rng.uniform(0.5, 1.0, host.res_scale[:, 1].shape) * 2.0 ** -10).astype(np.float16)
    cu, parent = make_tree([10, 4], "tree", rng)
    q, k, v = inputs(host, 14, rng, amp=0.1)
    v *= 2.0 ** -10
    for h in range(2):
        K = reconstruct(host, 0, 0, h, 0)[place]
        host.res_scale[0, 1, h, place] = 2.0 ** 15
        away = torch.from_numpy(K * (50.0 / (D ** -0.5 * 1.4427 * (K @ K)))).float()
        q[:10, 4 * h:4 * h + 4] -= away.to(q.dtype)
        q[[2, 7], 4 * h:4 * h + 4] += (2 * away).to(q.dtype)
        k[:10, h] = torch.from_numpy(K).half()          # the drafted keys are not looked at either
    announce(f"tree decode, a large value scale at {place} {fmt} {rb}")
    got = run(host, cu, parent, q, k, v)
    want, top = reference(host, 0, cu, parent, q.double().numpy(), k.double().numpy(), v.double().numpy())
    assert top < 100.0 and np.abs(want[[0, 1, 3, 4]]).max() < 1.0 < np.abs(want[[2, 7]]).max()
    check(got, want, bound(host, top), f"value scale at {place} {fmt} {rb}")


@pytest.mark.parametrize("rb", [16, 96])
@pytest.mark.parametrize("gap", [10, 18])
def test_probabilities_far_below_the_largest(gap, rb):
    """Tokens with empty values take most of the attention, in the first tile of every wave of one chunk; the other 16384
    tokens' probabilities are 2^-gap of theirs, and the row is theirs.  Scores are one product each, so the bound is
    tighter than random scores': S is kept to 2^-22 of 18 (3e-6 of a probability), float32 sums of 16384 terms of either
    sign to sqrt(16384) 2^-24 (7.6e-6), the 128 additions of a lane's sum of probabilities to 2^-17 (7.6e-6), and a
    probability of 2^-9, 18 binades below the largest, to 2^-25 / sqrt(3) of either sign (8.8e-6 of it): together 2.7e-5,
    below 2^-15."""
    torch = torch_gpu()
    lib_ready()
    T = 16384
    host = make_host([T], 4, rb, (0,))
    rng = np.random.default_rng(gap)
    host.basis[:, :, :, 0] = 0
    host.basis[:, :, :, 0, 0, 0] = 1
    host.coef_k[...] = 0
    host.coef_k[..., 0] = rng.uniform(0.0, 0.5, host.coef_k.shape[:-1])
    sinks = np.arange(0, 256, 32)
    host.coef_k[:, :, sinks, 0] = 32
    host.coef_v[:, :, sinks // 16, :, sinks % 16] = 0
    cu, parent = make_tree([3], "tree", rng)
    q, k, v = inputs(host, 3, rng)
    q[...] = 0
    q[..., 0] = 1
    k[...] = 0
    scale = gap * np.log(2.0) / 32
    announce(f"tree decode, probabilities 2^-{gap} of the largest, r_b {rb}")
    got = run(host, cu, parent, q, k, v, split=T, sm_scale=scale)
    want, _ = reference(host, 0, cu, parent, q.double().numpy(), k.double().numpy(), v.double().numpy(), scale=scale)
    check(got, want, 2.0 ** -15, f"probabilities 2^-{gap} of the largest, r_b {rb}")


@pytest.mark.parametrize("fmt", ["f16", "int8"])
def test_scores_that_are_no_numbers_reach_their_rows(fmt):
    """A key that is no number, as a sequence's one token and among others: every row of its sequence is no number, and no
    other row."""
    torch_gpu()
    lib_ready()
    host = make_host([1, 40, 700, 33], 4, 32, (0, 8), fmt=fmt)
    for t in (0, 1 + 40 + 300):
        (host.coef_scale_k[:, :, 0] if fmt == "int8" else host.coef_k[..., 0])[..., t] = np.nan
    rng = np.random.default_rng(3)
    cu, parent = make_tree([3, 5, 9, 4], "tree", rng)
    q, k, v = inputs(host, 21, rng)
    announce(f"tree decode, keys that are no numbers {fmt}")
    got = run(host, cu, parent, q, k, v)
    bad = np.zeros(21, bool)
    bad[:3] = bad[8:17] = True
    assert np.all(np.isnan(got[bad])) and np.all(np.isfinite(got[~bad]))


@pytest.mark.parametrize("fmt", ["f16", "int8"])
@pytest.mark.parametrize("amp", [0.3, 5.0])
def test_few_tokens_hold_all_the_values(amp, fmt):
    """A dozen of 3000 tokens have a value at all, a residual's, at scales from 2^-12 to 2^10 and probabilities far apart:
    each row is their sum, to the bound of its scores."""
    torch_gpu()
    lib_ready()
    host = make_host([3000, 50], 4, 32, (0, 4, 16), fmt=fmt)
    rng = np.random.default_rng(int(amp))
    host.coef_v[...] = 0
    rho = np.diff(host.res_off[0, 0].astype(np.int64))
    some = np.sort(rng.choice(np.nonzero(rho[:3000])[0], 12, replace=False))
    scale = np.zeros(host.res_scale[:, 1].shape, np.float16)
    scale[..., some] = 2.0 ** rng.uniform(-12, 10, scale[..., some].shape)
    host.res_scale[:, 1] = scale
    cu, parent = make_tree([9, 2], "tree", rng)
    q, k, v = inputs(host, 11, rng, amp=amp)
    v[...] = 0
    announce(f"tree decode, few values, amp {amp} {fmt}")
    got = run(host, cu, parent, q, k, v, split=1024)
    want, top = reference(host, 0, cu, parent, q.double().numpy(), k.double().numpy(), v.double().numpy())
    assert np.all(got[9:] == 0) and np.all(want[9:] == 0)
    check(got, want, bound(host, top), f"few values, amp {amp} {fmt}")
