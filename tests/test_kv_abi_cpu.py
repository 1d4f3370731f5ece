"""Host-only checks of the paged key-value cache's entry points: every refusal that the header states comes
before a device is touched."""
import ctypes as C

import pytest

from paper_2602_11688_b200 import binding as gb

A = 1 << 20                                # an aligned address that is never read


def cache(**kw):
    base = dict(k=A, v=2 * A, k_exp=None, v_exp=None, n_pages=8, page_tokens=16, n_kv_heads=2, head_dim=64,
                type=gb.GORGO_BF16, device=0)
    return gb.gorgo_kv_cache_t(**{**base, **kw})


def batch(**kw):
    base = dict(n_seqs=2, total_new=5, max_new=3, max_kv=40, total_kv=60, table_stride=3, reserved=0,
                cu_new=A, kv_len=A, table=A, status=None)
    return gb.gorgo_kv_batch_t(**{**base, **kw})


def calls(c, b, *, heads=4, type=gb.GORGO_BF16, stride=None, out_stride=None, p=A, scale=0.1, ws=4 << 30):
    """Status of every entry point for the same arguments (the four that take rows)."""
    lib = gb.load()
    kv = (c.n_kv_heads * c.head_dim if c else 128) if stride is None else stride
    qs = heads * (c.head_dim if c else 64) if stride is None else stride
    cp, bp = gb._struct_ptr(c), gb._struct_ptr(b)
    os = qs if out_stride is None else out_stride
    return {"write": lib.gorgo_kv_write(cp, bp, p, p, type, kv, kv, None),
            "read": lib.gorgo_kv_read(cp, bp, p, p, type, kv, kv, None),
            "prefill": lib.gorgo_attn_prefill(cp, bp, p, heads, type, qs, scale, p, os, None, A, ws, None),
            "decode": lib.gorgo_attn_decode(cp, bp, p, heads, type, qs, scale, p, os, None, A, ws, None)}


def test_an_empty_batch_is_fine_and_touches_nothing():
    assert set(calls(cache(), batch(n_seqs=0, cu_new=None, kv_len=None, table=None), p=None).values()) == {gb.GORGO_OK}
    got = calls(cache(), batch(total_new=0, max_new=0), p=None)
    assert got["write"] == got["read"] == got["prefill"] == gb.GORGO_OK
    rc, n = gb.gorgo_attn_workspace_bytes(cache(), batch(n_seqs=0), 4, gb.GORGO_BF16, 1)
    assert (rc, n) == (gb.GORGO_OK, 0)


@pytest.mark.parametrize("bad", [
    dict(k=None), dict(v=None), dict(k=A + 64), dict(type=3), dict(type=gb.GORGO_E4M3), dict(k_exp=A), dict(v_exp=A),
    dict(type=gb.GORGO_E4M3, k_exp=A, v_exp=A + 8), dict(n_pages=0), dict(page_tokens=0), dict(page_tokens=8),
    dict(page_tokens=48), dict(page_tokens=2048), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=96),
    dict(head_dim=256), dict(device=-1), dict(n_pages=1 << 26, page_tokens=16)])
def test_bad_caches_are_refused(bad):
    assert set(calls(cache(**bad), batch()).values()) == {gb.GORGO_ERR_INVALID_ARG}
    rc, _ = gb.gorgo_attn_workspace_bytes(cache(**bad), batch(), 4, gb.GORGO_BF16, 0)
    assert rc == gb.GORGO_ERR_INVALID_ARG


def test_sequences_without_tokens_need_no_table():
    got = calls(cache(), batch(total_new=0, max_new=0, max_kv=0, total_kv=0, table=None, table_stride=0), p=None)
    assert got["write"] == got["read"] == got["prefill"] == gb.GORGO_OK


@pytest.mark.parametrize("bad", [
    dict(reserved=1), dict(n_seqs=65536), dict(total_kv=1 << 40), dict(kv_len=None), dict(table=None), dict(table_stride=2), dict(max_kv=1 << 24)])
def test_bad_batches_are_refused(bad):
    assert set(calls(cache(), batch(**bad)).values()) == {gb.GORGO_ERR_INVALID_ARG}


@pytest.mark.parametrize("bad", [dict(cu_new=None), dict(max_new=6), dict(total_new=1 << 24)])
def test_bad_new_tokens_are_refused_where_they_are_used(bad):
    got = calls(cache(), batch(**bad))
    assert got["write"] == got["read"] == got["prefill"] == gb.GORGO_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(p=None), dict(p=A + 8), dict(stride=120), dict(stride=1 << 32),
                                dict(type=gb.GORGO_FP16), dict(type=gb.GORGO_E4M3)])
def test_bad_rows_are_refused(kw):
    assert set(calls(cache(), batch(), **kw).values()) == {gb.GORGO_ERR_INVALID_ARG}


@pytest.mark.parametrize("heads", [0, 3, 258])
def test_heads_are_a_multiple_of_the_kv_heads(heads):
    got = calls(cache(), batch(), heads=heads)
    assert got["prefill"] == got["decode"] == gb.GORGO_ERR_INVALID_ARG
    rc, _ = gb.gorgo_attn_workspace_bytes(cache(), batch(), heads, gb.GORGO_BF16, 1)
    assert rc == gb.GORGO_ERR_INVALID_ARG


@pytest.mark.parametrize("kw,code", [(dict(scale=float("nan")), gb.GORGO_ERR_NONFINITE_PARAM),
                                     (dict(scale=float("inf")), gb.GORGO_ERR_NONFINITE_PARAM),
                                     (dict(scale=1e39), gb.GORGO_ERR_NONFINITE_PARAM),
                                     (dict(out_stride=255), gb.GORGO_ERR_INVALID_ARG),
                                     (dict(out_stride=248), gb.GORGO_ERR_INVALID_ARG)])
def test_attention_refuses_bad_scales_and_outputs(kw, code):
    got = calls(cache(), batch(), **kw)
    assert got["prefill"] == got["decode"] == code


def test_prefill_refuses_a_16_bit_copy_of_too_many_rows():
    c = cache(type=gb.GORGO_E4M3, k_exp=A, v_exp=A, n_pages=1 << 20)
    b = batch(total_kv=1 << 30)
    assert calls(c, b)["prefill"] == gb.GORGO_ERR_INVALID_ARG
    assert gb.gorgo_attn_workspace_bytes(c, b, 4, gb.GORGO_BF16, 0)[0] == gb.GORGO_ERR_INVALID_ARG


def test_null_structures_are_refused():
    assert set(calls(None, batch()).values()) == {gb.GORGO_ERR_INVALID_ARG}
    assert set(calls(cache(), None).values()) == {gb.GORGO_ERR_INVALID_ARG}
    assert gb.load().gorgo_attn_workspace_bytes(C.addressof(cache()), C.addressof(batch()), 4, 0, 1, None) == \
        gb.GORGO_ERR_INVALID_ARG


@pytest.mark.parametrize("what", ["kv_len", "table", "status", "cu_new"])
@pytest.mark.parametrize("off", [1, 2, 3])
def test_arrays_that_are_not_aligned_to_their_elements_are_refused(what, off):
    got = calls(cache(), batch(**{what: A + off}))
    assert got["write"] == got["read"] == got["prefill"] == gb.GORGO_ERR_INVALID_ARG
    if what != "cu_new":
        assert got["decode"] == gb.GORGO_ERR_INVALID_ARG


@pytest.mark.parametrize("decode", [False, True])
def test_an_lse_that_is_not_aligned_is_refused(decode):
    lib, c, b = gb.load(), cache(), batch()
    f = lib.gorgo_attn_decode if decode else lib.gorgo_attn_prefill
    assert f(C.addressof(c), C.addressof(b), A, 4, gb.GORGO_BF16, 256, 0.1, A, 256, A + 2, A, 4 << 30, None) == \
        gb.GORGO_ERR_INVALID_ARG
