"""The longest sequence of a 4-bit pool (32-bit row numbers reach it: 146 GB at one head of 64)."""
import pytest

LONGEST = 2 ** 31 - 256


def test_rows_beyond_32_bits_are_refused(stlib):
    """Bookkeeping alone; in every appending call, without a change."""
    n_blocks = 2 ** 27 + 16
    pool = stlib.Pool(n_layers=1, n_q_heads=1, n_kv_heads=1, head_dim=64, n_blocks=n_blocks, max_seqs=2, device=None,
                      kv_bits=4)
    s = pool.seq_create()
    pool.append_kv([s], 2 ** 30, None)
    pool.append_kv([s], 2 ** 30 - 257, None)
    other = pool.seq_create()
    for call in (lambda: pool.append_kv([s], 2, None), lambda: pool.merge(s, 2, None, None),
                 lambda: pool.prefill_batch([other, s], [1, 2], None, None, None),
                 lambda: pool.append_kv([s], 2 ** 31 - 1, None)):
        with pytest.raises(stlib.STError) as e:
            call()
        assert e.value.status == stlib.ST_ERR_OOM
    pool.merge(s, 1, None, None)
    with pytest.raises(stlib.STError):
        pool.append_kv([s], 1, None)
    items, _, _ = pool.decode_plan([s])
    assert sum(i["n_tokens"] for i in items) == LONGEST
    assert all(0 < i["n_tokens"] <= i["n_pages"] * 16 < 2 ** 31 for i in items)
    pool.close()
