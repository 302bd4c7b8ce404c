"""What the profile counts of a 4-bit pool's calls: launches, and bytes beyond the algorithmic ones."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def zeros(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16, device="cuda")


def make(stlib, L=2, Hkv=2, G=8, **kw):
    return stlib.Pool(n_layers=L, n_q_heads=G * Hkv, n_kv_heads=Hkv, head_dim=128, n_blocks=600, max_seqs=40,
                      max_decode_branches=32, kv_bits=4, **kw)


@pytest.mark.parametrize("branches", [[3], [12], [12, 5], [20, 1, 6]])
def test_a_decode_is_one_launch_and_its_combine(stlib, branches):
    """Narrow and wide groups of a call go out together."""
    pool, br = make(stlib), []
    for i, n in enumerate(branches):
        m = pool.seq_create()
        ctx = 300 + 500 * i
        pool.append_kv([m], zeros(2, 1, ctx, 2, 128), zeros(2, 1, ctx, 2, 128))
        br += [m] + pool.fork(m, n - 1)
    pool.append_kv(br, zeros(2, len(br), 1, 2, 128), zeros(2, len(br), 1, 2, 128))
    pool.sync()
    pool.profile_read()
    pool.decode_attn(br, zeros(2, len(br), 16, 128))
    got = pool.profile_read()
    assert got["decode_partial"]["kernels"] == 1 and got["lse_combine"]["kernels"] == 1


def test_a_small_append_counts_its_tables_and_copied_rows(stlib):
    pool = make(stlib)
    token = 2 * 2 * 2 * (1088 // 16)  # layers, KV heads, K and V
    m = pool.seq_create()
    pool.profile_read()
    pool.append_kv([m], zeros(2, 1, 165, 2, 128), zeros(2, 1, 165, 2, 128))
    got = pool.profile_read()["append_kv"]
    assert got["kernels"] == 1 and got["overhead_bytes"] == 11 * 8 + 16  # 11 entries, one range
    pool.append_kv([m], zeros(2, 1, 3, 2, 128), zeros(2, 1, 3, 2, 128))
    assert pool.profile_read()["append_kv"]["overhead_bytes"] == 0
    f, = pool.fork(m, 1)
    pool.append_kv([f], zeros(2, 1, 1, 2, 128), zeros(2, 1, 1, 2, 128))
    got = pool.profile_read()["append_kv"]  # the table of a fork goes out whole; 8 rows of its last page copied
    assert got["kernels"] == 1 and got["overhead_bytes"] == 8 * token * 2 + 11 * 8 + 16
