"""How large a call of attention over the 4-bit cache may be: the limits that include/sjd.h names, from both sides, through the call that plans it (CPU)."""
import ctypes as C

import pytest

import paper_2505_24791_amd as sjd

F16, BF16, F32 = sjd.DTYPE_F16, sjd.DTYPE_BF16, sjd.DTYPE_F32


def _planned(*, dtype=BF16, kv=1, heads=1, dim=64, n_seqs=1, n_rows=None, max_q=1, max_kv=4096, max_pages=None, ragged=False):
    """(return code, message, bytes of workspace)"""
    cache = sjd.SjdKv4(None, 4, kv, dim, dtype)
    n_rows = n_seqs * max_q if n_rows is None else n_rows
    pages = -(-max_kv // 64) if max_pages is None else max_pages
    a = sjd.SjdKv4Attention(None, None, heads * dim, heads * dim, pages, 0x10000 if ragged else None, None, None, n_seqs, heads, n_rows, pages,
                            max_q, max_kv, 1, 0, 0, 0.1, None, 0)
    lib, need = sjd.load_library(), C.c_size_t()
    rc = lib.sjd_kv4_attention_workspace(C.addressof(cache), C.addressof(a), C.addressof(need))
    return rc, lib.sjd_last_error().decode() if rc else "", need.value


@pytest.mark.parametrize("dtype,kv,heads,dim,rows", [
    (BF16, 1, 16, 128, 131072), (F32, 1, 8, 128, 131072), (BF16, 1, 8, 256, 131072), (F16, 2, 2, 64, 2 ** 22), (F32, 1, 1, 32, 2 ** 24), (F16, 8, 64, 128, 2 ** 20)])
def test_a_long_prompt_is_one_call(dtype, kv, heads, dim, rows):
    """More than 65535 row tiles, of 16 and of 32 rows."""
    assert _planned(dtype=dtype, kv=kv, heads=heads, dim=dim, max_q=rows, max_kv=rows) == (sjd.SJD_OK, "", 0)


@pytest.mark.parametrize("dtype", [F32, F16])
@pytest.mark.parametrize("inside,outside", [
    (dict(n_seqs=65535), dict(n_seqs=65536)),
    (dict(max_kv=2 ** 30 - 1), dict(max_kv=2 ** 30)),
    (dict(max_pages=2 ** 25 - 1), dict(max_pages=2 ** 25)),
    (dict(max_q=2 ** 30 - 1), dict(max_q=2 ** 30)),                                                          # max_q * n_heads
    (dict(kv=2, heads=2, max_q=2 ** 29 - 1), dict(kv=2, heads=2, max_q=2 ** 29)),
    (dict(heads=64, max_q=2 ** 19 - 1), dict(heads=64, max_q=2 ** 19)),                                      # max_q * group^2
    (dict(n_seqs=5, kv=2, heads=2, max_q=214748364), dict(n_seqs=5, kv=2, heads=2, max_q=214748365)),        # n_seqs * n_heads * max_q
    (dict(n_seqs=65535, n_rows=32768, max_q=32768, ragged=True), dict(n_seqs=65535, n_rows=32769, max_q=32769, ragged=True)),
    (dict(n_rows=5, max_q=2 ** 31 - 1, ragged=True), None)])                                                 # no more rows than there are
def test_limits_from_both_sides(dtype, inside, outside):
    rc, message, _ = _planned(dtype=dtype, **inside)
    assert rc == sjd.SJD_OK, message
    if outside:
        rc, message, _ = _planned(dtype=dtype, **outside)
        assert rc == sjd.SJD_EINVAL and ("out of range" in message or "too many" in message)
