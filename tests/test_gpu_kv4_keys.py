"""Every key counts once: queries along single keys, at the borders of pages, stages of 128, runs,
splits and causal limits, so that a key that is lost, read twice or seen too early shows at any
length (kv4_close.py; test_kv4_tolerance.py tests that it does)."""
import pytest
import torch

from kv4_close import check, held

pytestmark = pytest.mark.gpu


def drawn(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def along(k, at):
    """Queries [len(at), D] that look for keys k[at] ([n, D])."""
    return (k[at].float() * (1.0 if k.shape[1] == 128 else 1.5)).bfloat16()


def fill(pool, s, k, v, piece=1 << 16):
    for i in range(0, k.shape[0], piece):
        pool.append_kv([s], k[None, None, i:i + piece].contiguous().cuda(), v[None, None, i:i + piece].contiguous().cuda())


def borders(n, items, members, branch):
    """Keys at either side of every run's ends, of page and stage borders near the end and the beginning."""
    at = {0, 1, n - 2, n - 1}
    for it in items:
        if branch in members[it["member_base"]:it["member_base"] + it["n_members"]]:
            first = it["page_begin"] * 16
            at |= {first - 1, first, first + 1, first + 127, first + 128, first + it["n_tokens"] - 1, first + it["n_tokens"]}
    for x in (16, 128, n // 128 * 128, n // 16 * 16):
        at |= {x - 1, x}
    return sorted(x for x in at if 0 <= x < n)


def probe_decode(pool, br, contexts, Hq, what):
    """Decodes in which every query row looks for a key of its branch's own borders, until all have been looked for."""
    D = contexts[0][0].shape[2]
    items, members, _ = pool.decode_plan(br)
    todo = [borders(k.shape[0], items, members, i) for i, (k, _) in enumerate(contexts)]
    g = Hq // contexts[0][0].shape[1]
    for r in range(0, max(len(x) for x in todo), Hq):
        q = torch.empty(len(br), Hq, D, dtype=torch.bfloat16)
        for i, (k, _) in enumerate(contexts):
            for h in range(Hq):
                q[i, h] = along(k[:, h // g], [todo[i][(r + h) % len(todo[i])]])[0]
        o, lse = pool.decode_attn(br, q[None].cuda())
        pool.sync()
        check(o[0], lse[0], q, contexts, f"{what}, round {r}")


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 1), (64, 16, 2)])
@pytest.mark.parametrize("n", [17, 129, 2049, 5000, 9001])
@pytest.mark.parametrize("branches", [1, 5, 18])
def test_decode_at_the_borders_of_runs(stlib, D, Hq, Hkv, n, branches):
    """A lone sequence, a narrow group, and subgroups of a wide one with pages of their own."""
    pool = stlib.Pool(n_layers=1, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, n_blocks=n // 16 + 400, max_seqs=20,
                      max_decode_branches=18, kv_bits=4)
    k, v = drawn(n, Hkv, D, seed=n).bfloat16(), drawn(n, Hkv, D, seed=n + 1).bfloat16()
    m = pool.seq_create()
    fill(pool, m, k, v)
    hk, hv = held(k), held(v)
    br, contexts = [m] + pool.fork(m, branches - 1), [(hk, hv)] * branches
    for i in range(0, branches if branches > 1 else 0, 3):
        T = 1 + 67 * i % 190
        nk, nv = drawn(T, Hkv, D, seed=50 + i).bfloat16(), drawn(T, Hkv, D, seed=90 + i).bfloat16()
        pool.append_kv([br[i]], nk[None, None].cuda(), nv[None, None].cuda())
        contexts[i] = torch.cat([hk, held(nk)]), torch.cat([hv, held(nv)])
    probe_decode(pool, br, contexts, Hq, f"n {n}")


@pytest.mark.parametrize("max_splits", [2, 7, 32])
def test_decode_at_the_borders_of_a_split_budget(stlib, max_splits):
    n, D = 7000, 128
    pool = stlib.Pool(n_layers=1, n_q_heads=8, n_kv_heads=1, head_dim=D, n_blocks=600, max_seqs=4, max_splits=max_splits,
                      kv_bits=4)
    k, v = drawn(n, 1, D, seed=1).bfloat16(), drawn(n, 1, D, seed=2).bfloat16()
    m = pool.seq_create()
    fill(pool, m, k, v)
    probe_decode(pool, [m] + pool.fork(m, 2), [(held(k), held(v))] * 3, 8, f"{max_splits} splits")


def probe_prefill(pool, s, k, v, n, T, Hq, what, rows):
    """The T rows behind the first n of k, v merged onto s; row t's heads look in turn for itself, the row behind
    it (which it must not see), the one before it and keys at stage borders."""
    D = k.shape[2]
    g = Hq // k.shape[1]
    q = torch.empty(T, Hq, D, dtype=torch.bfloat16)
    stages = [x for b in range(128, n + T, 128) for x in (b - 1, b)] + [0, max(0, n - 1)]
    for t in range(T):
        for h in range(Hq):
            # no query looks for a key that it does not see, but for the one behind it
            own = [n + t, min(n + t + 1, n + T - 1), max(0, n + t - 1)]
            pick = own[h % 4] if h % 4 < 3 else min(stages[(t * Hq + h) // 4 % len(stages)], n + t)
            q[t, h] = along(k[:, h // g], [pick])[0]
    o, lse = pool.merge(s, q[None].cuda(), k[None, n:].contiguous().cuda(), v[None, n:].contiguous().cuda())
    pool.sync()
    hk, hv = held(k), held(v)
    check(o[0][rows], lse[0][rows], q[rows], [(hk[:n + t + 1], hv[:n + t + 1]) for t in rows], what)


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 1), (64, 8, 2)])
@pytest.mark.parametrize("n,T", [(0, 300), (100, 5), (127, 2), (1000, 33), (3900, 40), (4000, 8), (9000, 133)])
def test_prefill_at_the_borders_of_splits(stlib, D, Hq, Hkv, n, T):
    pool = stlib.Pool(n_layers=1, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, n_blocks=(n + T) // 16 + 20, max_seqs=2,
                      kv_bits=4)
    k, v = drawn(n + T, Hkv, D, seed=n + T).bfloat16(), drawn(n + T, Hkv, D, seed=n + T + 1).bfloat16()
    s = pool.seq_create()
    if n:
        fill(pool, s, k[:n], v[:n])
    rows = sorted({0, 1, T - 2, T - 1} & set(range(T)) | set(range(0, T, max(1, T // 24))))
    probe_prefill(pool, s, k, v, n, T, Hq, f"{T} rows onto {n}", rows)


# ---- at the length that the sums' tolerance is stated for ------------------------------------


@pytest.mark.parametrize("D,Hq", [(128, 8), (64, 4)])
def test_long_decode(stlib, D, Hq):
    """131072 keys and some: runs of many stages, branches with rows of their own."""
    n = 131072 + 77
    pool = stlib.Pool(n_layers=1, n_q_heads=Hq, n_kv_heads=1, head_dim=D, n_blocks=n // 16 + 200, max_seqs=6, kv_bits=4)
    k, v = drawn(n, 1, D, seed=7).bfloat16(), drawn(n, 1, D, seed=8).bfloat16()
    m = pool.seq_create()
    fill(pool, m, k, v)
    hk, hv = held(k), held(v)
    br, contexts = [m] + pool.fork(m, 4), [(hk, hv)] * 5
    for i in (1, 3):
        nk, nv = drawn(200 * i, 1, D, seed=20 + i).bfloat16(), drawn(200 * i, 1, D, seed=30 + i).bfloat16()
        fill(pool, br[i], nk, nv)
        contexts[i] = torch.cat([hk, held(nk)]), torch.cat([hv, held(nv)])
    probe_decode(pool, br, contexts, Hq, "long")
    q = drawn(1, 5, Hq, D, seed=9).bfloat16()
    o, lse = pool.decode_attn(br, q.cuda())
    pool.sync()
    check(o[0], lse[0], q[0], contexts, "long, drawn queries")


@pytest.mark.parametrize("T", [5, 40])
def test_long_prefill(stlib, T):
    """Narrow and wide tiles, each split over the keys."""
    n, D, Hq = 131072 - 19, 128, 8
    pool = stlib.Pool(n_layers=1, n_q_heads=Hq, n_kv_heads=1, head_dim=D, n_blocks=n // 16 + 20, max_seqs=2, kv_bits=4)
    k, v = drawn(n + T, 1, D, seed=17).bfloat16(), drawn(n + T, 1, D, seed=18).bfloat16()
    s = pool.seq_create()
    fill(pool, s, k[:n], v[:n])
    pool.profile_read()
    probe_prefill(pool, s, k, v, n, T, Hq, "long", sorted({0, T // 2, T - 1}))
    assert pool.profile_read()["merge_prefill"]["kernels"] == 2
