"""Calls of the attention whose join would need more workgroups than are numbered (2^31), on the CPU."""
import ctypes

import pytest

from paper_2504_00598_amd import _lib as L
from paper_2504_00598_amd import block as B
from tests.test_block_cache_host import P, cache, queries, seqs

ref = ctypes.byref


@pytest.mark.parametrize("n_seqs,group,code", [
    # 64 key heads of dim 256: 64 * 16 rows * 64 quads / 32 = 2048 workgroups a sequence, 4096 for 32 rows
    ((1 << 20), 16, L.CFP_ERR_UNSUPPORTED), ((1 << 20), 32, L.CFP_ERR_UNSUPPORTED), ((1 << 19), 32, L.CFP_ERR_UNSUPPORTED),
    ((1 << 19) + 1, 32, L.CFP_ERR_UNSUPPORTED), ((1 << 20) - 1, 16, L.CFP_ERR_WORKSPACE), ((1 << 19) - 1, 32, L.CFP_ERR_WORKSPACE),
    ((1 << 20), 8, L.CFP_ERR_WORKSPACE)])
def test_more_joins_than_workgroups(n_seqs, group, code):
    c = ref(cache(heads=64, dim=256, k_page_stride=1 << 18, v_page_stride=1 << 18))
    s = ref(seqs(n_seqs=n_seqs, width=64, table_stride=64, max_new=1))
    a = ref(queries(n_tokens=1 << 17, n_q=64 * group, q_token_stride=64 * group * 256, q_head_stride=256))
    need = B.lib().cfp_attend_workspace_bytes(a, c, s)
    assert (need > 0) == (code == L.CFP_ERR_WORKSPACE)
    assert B.lib().cfp_attend(a, c, s, P, P, None, 0, None) == code
