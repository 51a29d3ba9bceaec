"""The operators over a paged cache and rotation by several axes on the CPU: what they refuse before they touch a device."""
import ctypes

import pytest

from paper_2504_00598_amd import _lib as L
from paper_2504_00598_amd import block as B

P = 0x1000  # a pointer that no refused call follows
ref = ctypes.byref


def cache(**kw):
    d = dict(n_pages=8, page=16, heads=2, dim=32, dtype=2, k=P, v=P, k_scale=None, v_scale=None, k_page_stride=1024,
             v_page_stride=1024, k_scale_page_stride=0, v_scale_page_stride=0)
    d.update(kw)
    return B.cfp_cache_desc(**d)


def seqs(**kw):
    d = dict(n_seqs=3, width=4, table=P, table_stride=4, starts=P, lengths=P, max_new=5)
    d.update(kw)
    return B.cfp_sequences_desc(**d)


def queries(**kw):
    d = dict(n_tokens=9, n_q=4, dtype=2, q=P, q_token_stride=128, q_head_stride=32, scale=0.2, causal=1, window=0)
    d.update(kw)
    return B.cfp_attend_desc(**d)


def calls(c, s, a, n=9, dtype=2):
    """Return codes of the three operators."""
    lib = B.lib()
    return (lib.cfp_cache_write(c, s, n, dtype, P, 64, 32, P, 64, 32, None), lib.cfp_cache_read(c, s, n, dtype, P, P, None),
            lib.cfp_attend(a, c, s, P, P, P, 1 << 50, None))


BYTE = dict(dtype=3, k_scale=P, v_scale=P, k_scale_page_stride=32, v_scale_page_stride=32)


@pytest.mark.parametrize("bad,code", [
    (dict(n_pages=0), L.CFP_ERR_ARG), (dict(page=0), L.CFP_ERR_ARG), (dict(heads=0), L.CFP_ERR_ARG),
    (dict(dim=0), L.CFP_ERR_ARG), (dict(dtype=0), L.CFP_ERR_ARG), (dict(dtype=4), L.CFP_ERR_ARG), (dict(k=None), L.CFP_ERR_ARG),
    (dict(v=None), L.CFP_ERR_ARG), (dict(k=P + 8), L.CFP_ERR_ARG), (dict(v=P + 2), L.CFP_ERR_ARG),
    (dict(k_page_stride=1023), L.CFP_ERR_ARG), (dict(v_page_stride=1008), L.CFP_ERR_ARG),
    (dict(k_page_stride=1032), L.CFP_ERR_ARG), (dict(v_page_stride=-1024), L.CFP_ERR_ARG),
    (dict(page=8), L.CFP_ERR_UNSUPPORTED), (dict(page=48), L.CFP_ERR_UNSUPPORTED), (dict(page=512), L.CFP_ERR_UNSUPPORTED),
    (dict(dim=40), L.CFP_ERR_UNSUPPORTED), (dict(dim=272), L.CFP_ERR_UNSUPPORTED), (dict(n_pages=1 << 31), L.CFP_ERR_UNSUPPORTED),
    (dict(heads=1 << 24), L.CFP_ERR_UNSUPPORTED), (dict(dtype=3), L.CFP_ERR_ARG), (dict(BYTE, v_scale=None), L.CFP_ERR_ARG),
    (dict(BYTE, k_scale=P + 4), L.CFP_ERR_ARG), (dict(BYTE, k_scale_page_stride=24), L.CFP_ERR_ARG),
    (dict(BYTE, v_scale_page_stride=40), L.CFP_ERR_ARG)])
def test_caches_refused(bad, code):
    assert calls(ref(cache(**bad)), ref(seqs()), ref(queries())) == (code,) * 3


@pytest.mark.parametrize("bad,code", [
    (dict(n_seqs=-1), L.CFP_ERR_ARG), (dict(width=-1), L.CFP_ERR_ARG), (dict(table=None), L.CFP_ERR_ARG),
    (dict(starts=None), L.CFP_ERR_ARG), (dict(lengths=None), L.CFP_ERR_ARG), (dict(table_stride=3), L.CFP_ERR_ARG),
    (dict(max_new=-1), L.CFP_ERR_ARG), (dict(width=1 << 26, table_stride=1 << 26), L.CFP_ERR_UNSUPPORTED),
    (dict(n_seqs=(1 << 31) - 1), L.CFP_ERR_UNSUPPORTED)])
def test_sequences_refused(bad, code):
    assert calls(ref(cache()), ref(seqs(**bad)), ref(queries())) == (code,) * 3


@pytest.mark.parametrize("bad,code", [
    (dict(n_tokens=-1), L.CFP_ERR_ARG), (dict(n_q=0), L.CFP_ERR_ARG), (dict(n_q=3), L.CFP_ERR_ARG), (dict(q=None), L.CFP_ERR_ARG),
    (dict(dtype=0), L.CFP_ERR_ARG), (dict(dtype=3), L.CFP_ERR_ARG), (dict(dtype=1), L.CFP_ERR_UNSUPPORTED),
    (dict(scale=0.0), L.CFP_ERR_ARG), (dict(scale=-1.0), L.CFP_ERR_ARG), (dict(scale=float("nan")), L.CFP_ERR_ARG),
    (dict(scale=float("inf")), L.CFP_ERR_ARG), (dict(window=-1), L.CFP_ERR_ARG), (dict(n_tokens=1 << 31), L.CFP_ERR_UNSUPPORTED),
    (dict(n_tokens=1 << 29), L.CFP_ERR_UNSUPPORTED), (dict(n_q=1 << 30), L.CFP_ERR_UNSUPPORTED)])
def test_queries_refused(bad, code):
    assert calls(ref(cache()), ref(seqs()), ref(queries(**bad)))[2] == code
    assert B.lib().cfp_attend_workspace_bytes(ref(queries(**bad)), ref(cache()), ref(seqs())) == 0


def test_rows_refused():
    lib, c, s = B.lib(), ref(cache()), ref(seqs())
    for n, dtype, code in ((-1, 2, L.CFP_ERR_ARG), (9, 0, L.CFP_ERR_ARG), (9, 3, L.CFP_ERR_ARG), (9, 1, L.CFP_ERR_UNSUPPORTED),
                           (1 << 31, 2, L.CFP_ERR_UNSUPPORTED), (1 << 30, 2, L.CFP_ERR_UNSUPPORTED)):
        assert calls(c, s, ref(queries()), n, dtype)[:2] == (code,) * 2
    assert lib.cfp_cache_write(c, s, 9, 2, None, 64, 32, P, 64, 32, None) == L.CFP_ERR_ARG
    assert lib.cfp_cache_write(c, s, 9, 2, P, 64, 32, None, 64, 32, None) == L.CFP_ERR_ARG
    assert lib.cfp_cache_read(c, s, 9, 2, P, None, None) == L.CFP_ERR_ARG
    assert lib.cfp_cache_read(c, s, 9, 2, P + 2, P, None) == L.CFP_ERR_ARG
    for args in ((None, s, ref(queries())), (c, None, ref(queries()))):
        assert calls(*args) == (L.CFP_ERR_ARG,) * 3
    assert lib.cfp_attend(None, c, s, P, P, P, 1 << 50, None) == L.CFP_ERR_ARG
    assert lib.cfp_attend(ref(queries()), c, s, None, P, P, 1 << 50, None) == L.CFP_ERR_ARG
    assert lib.cfp_attend(ref(queries()), c, s, P + 8, P, P, 1 << 50, None) == L.CFP_ERR_ARG


def test_nothing_to_do_is_no_error():
    for c in (cache(), cache(**BYTE)):
        assert calls(ref(c), ref(seqs()), ref(queries(n_tokens=0)), 0) == (L.CFP_OK,) * 3
        assert calls(ref(c), ref(seqs(n_seqs=0)), ref(queries())) == (L.CFP_OK,) * 3


def test_attend_workspace():
    lib, c, s = B.lib(), ref(cache()), ref(seqs(width=1000, table_stride=1000))
    a = ref(queries())
    need = lib.cfp_attend_workspace_bytes(a, c, s)
    assert need > 0
    assert lib.cfp_attend(a, c, s, P, P, P, need - 1, None) == L.CFP_ERR_WORKSPACE
    assert lib.cfp_attend(a, c, s, P, P, None, need, None) == L.CFP_ERR_WORKSPACE
    assert lib.cfp_attend(a, c, s, P, P, P + 8, need, None) == L.CFP_ERR_ARG
    assert lib.cfp_attend_workspace_bytes(a, c, ref(seqs(width=1))) == 0  # 16 tokens are one part


def test_axes_refused():
    d = dict(n_tokens=4, n_q=2, n_k=1, dim=8, rot=8, interleaved=0, dtype=2, wdtype=2, eps=1e-6, n_pos=16, q=P, k=P,
             q_token_stride=24, q_head_stride=8, k_token_stride=24, k_head_stride=8, wq=P, wk=P, cos=P, sin=P, pos=P)
    lib = B.lib()

    def codes(axis, n, **kw):
        q = B.cfp_qk_desc(**{**d, **kw})
        return {lib.cfp_qk_norm_rope_axes(ref(q), axis, n, P, P, None),
                lib.cfp_qk_norm_rope_axes_bwd(ref(q), axis, n, P, 24, 8, P, 24, 8, P, P, P, P, P, 1 << 20, None)}

    ok = bytes([0, 1, 2, 0])
    assert codes(ok, 2) == codes(ok, 0) == codes(ok, -1) == codes(None, 3) == codes(ok, 3, pos=None) == {L.CFP_ERR_ARG}
    assert codes(ok, 3, rot=6, dim=5) == codes(ok, 3, cos=None) == codes(ok, 3, eps=-1.0) == {L.CFP_ERR_ARG}
    assert codes(ok, 5) == {L.CFP_ERR_UNSUPPORTED}


def test_packed_descriptors_have_the_structures_layout():
    for pack, c in ((B._CACHE, B.cfp_cache_desc), (B._SEQUENCES, B.cfp_sequences_desc), (B._ATTEND, B.cfp_attend_desc)):
        values = [i + 1 for i, _ in enumerate(c._fields_)]
        packed = pack(*values)
        assert len(packed) == ctypes.sizeof(c)
        got = c.from_buffer_copy(packed)
        assert [getattr(got, f) for f, _ in c._fields_] == values


def test_the_binding_refuses_cpu_tensors():
    import torch
    k, v = torch.zeros(2, 1, 16, 32, dtype=torch.bfloat16), torch.zeros(2, 1, 32, 16, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        B.KVCache(k, v)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        B.Sequences(i[None], i, i[:1])
    for call in (lambda: B.attend(k[0], k, i), lambda: B.cache_write(k, k[0], k[0], i), lambda: B.cache_read(k, i, 1)):
        with pytest.raises(TypeError):
            call()
