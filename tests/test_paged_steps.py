"""Prompts and single steps over the paged cache, each sequence checked by itself: what the pages and
the turned queries hold against the inputs turned in 64 bits with one rounding, and the
attention against 64 bits over exactly those numbers.  The check is tried on the host with mistakes
planted in what it is given."""
import numpy as np
import pytest

from serving_ref import attend, check, key_rows, rotate, rounding, value_rows

H, G, D, PAGE = 2, 4, 64, 16
PROMPTS, STEPS = [37, 1, 64], 5


def of_sequence(pages, table, b, n):
    """Rows [n, H, d] of sequence b's tokens in pages [n_pages, H, page, d]."""
    return np.stack([pages[table[b, t // PAGE], :, t % PAGE] for t in range(n)])


def check_sequence(b, keys, values, query, freq, k_pages, v_pages, table, turned, out):
    """Everything of sequence b after a step: its rows keys and values [n, H, d] as they went in and its newest
    token's query [Hq, d], all bfloat16 numbers; the library's pages [n_pages, H, page, d], turned query and output."""
    n = len(keys)
    want, tol = rotate(keys, np.arange(n), freq, True)
    check(of_sequence(k_pages, table, b, n), want, tol + rounding(np.abs(want) + tol, "bf16"), f"stored keys of {b}")
    assert (of_sequence(v_pages, table, b, n) == values).all(), f"stored values of {b}"
    want, tol = rotate(query[None], [n - 1], freq, True)
    check(turned[None], want, tol + rounding(np.abs(want) + tol, "bf16"), f"query of {b}")
    want, tol = attend(turned[None], k_pages, v_pages, table[b:b + 1], [n])
    check(out[None], want, tol, f"attention of {b}")


def frequencies():
    from paper_2607_06523_amd import rope_freqs
    return rope_freqs(32, base=500000.0, scaling="linear", factor=2.0)


@pytest.mark.gpu
def test_steps():
    from gpu_util import announce, lib_ready, torch_gpu
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import PagedCache, RopeTable
    announce("paged steps")
    B, Hq, layer = len(PROMPTS), H * G, 1
    g = torch.Generator().manual_seed(0)
    draw = lambda n: torch.randn((n, Hq + 2 * H, D), generator=g).bfloat16().cuda()
    split = lambda x: (x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:])
    host = lambda x: x.double().cpu().numpy()
    table = torch.from_numpy(np.random.default_rng(0).permutation(24).astype(np.int32).reshape(B, 8)).cuda()
    lens = torch.tensor(PROMPTS, dtype=torch.int32, device="cuda")
    cache = PagedCache.empty(table, lens, n_pages=24, page_size=PAGE, n_kv_heads=H, n_q_heads=Hq, head_dim=D, n_layers=2, dtype=torch.bfloat16)
    freq = frequencies()
    rope = RopeTable(freq, interleaved=True)
    q, k, v = split(draw(sum(PROMPTS)))
    cu = np.concatenate([[0], np.cumsum(PROMPTS)])
    cache.append(layer, k, v, cu_new=torch.from_numpy(cu.astype(np.int32)).cuda(), q=q, rope=rope)
    keys, values = ([x[cu[b]:cu[b + 1]] for b in range(B)] for x in (host(k), host(v)))
    for _ in range(STEPS):
        lens += 1
        q, k, v = split(draw(B))
        turned = cache.append(layer, k, v, q=q, rope=rope)
        out = host(cache.decode(layer, turned))
        pages = key_rows(host(cache.k[layer])), value_rows(host(cache.v[layer]))
        for b in range(B):
            keys[b], values[b] = np.concatenate([keys[b], host(k)[b:b + 1]]), np.concatenate([values[b], host(v)[b:b + 1]])
            check_sequence(b, keys[b], values[b], host(q)[b], freq.numpy(), *pages, table.cpu().numpy(), host(turned)[b], out[b])


def rounded(x, to):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).to(to).double().numpy()


def step_on_the_host(keys, values, query, freq, table, n_pages, scaled=1.0, turn=True, pairs=True, drop=0, other_page=False, raw_query=False):
    """What the library gives for one sequence, in 64 bits rounded once; and with mistakes: frequencies off by
    a factor, no rotation, the wrong pairs, tokens dropped at the end, a page that is not the sequence's,
    a query that is attended with before its rotation."""
    import torch
    n = len(keys)
    spin = lambda x, pos: rounded(rotate(x, pos, freq * scaled, pairs)[0] if turn else x, torch.bfloat16)
    K, V = np.zeros((n_pages, H, PAGE, D)), np.zeros((n_pages, H, PAGE, D))
    turned = spin(query[None], [n - 1])[0]
    k = spin(keys, np.arange(n))
    for t in range(n):
        K[table[0, t // PAGE], :, t % PAGE], V[table[0, t // PAGE], :, t % PAGE] = k[t], values[t]
    read = table.copy()
    if other_page:
        read[0, 0] = table[0, -1]
    out = attend((query if raw_query else turned)[None], K, V, read, [n - drop])[0][0]
    return K, V, turned, rounded(out, torch.float32)


@pytest.mark.parametrize("n", [2, 6, 38, 42, 65, 69])
def test_the_check_sees_mistakes(n):
    import torch
    rng = np.random.default_rng(n)
    row = lambda *s: rounded(rng.normal(0, 1, s), torch.bfloat16)
    keys, values, query = row(n, H, D), row(n, H, D), row(H * G, D)
    table, freq = rng.permutation(8).astype(np.int32)[None], frequencies().numpy()

    def run(**mistake):
        K, V, turned, out = step_on_the_host(keys, values, query, freq, table, 8, **mistake)
        check_sequence(0, keys, values, query, freq, K, V, table, turned, out)
    run()
    mistakes = [dict(scaled=2.0), dict(scaled=1.25), dict(turn=False), dict(pairs=False), dict(drop=1), dict(raw_query=True),
                dict(other_page=True)]
    for m in mistakes:
        with pytest.raises(AssertionError):
            run(**m)
