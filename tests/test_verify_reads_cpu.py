"""Which rows of the draft's logits the verification may read, by the rule that its kernels
use: rows without a draft have none."""
import ctypes as C
import os

import pytest

torch = pytest.importorskip("torch")
from paper_2607_24841_amd import binding as B  # noqa: E402


@pytest.mark.parametrize("V", [1, 7, 32000, 1 << 24])
def test_draft_logits_of_rows_without_a_draft_are_not_read(V):
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libnmdlm.so not built")
    f = B.load().nmdlm_internal_draft_logits
    f.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int32]
    f.restype = C.c_void_p
    target, drafts = 1 << 45, 1 << 46   # never dereferenced
    for m in (0, 1, 8, 65534):
        for x in (-1, -2 ** 31, V, V + 1, 2 ** 31 - 1):
            assert f(target, drafts, m, V, x) == target + 4 * m * V
        for x in (0, V // 2, V - 1):
            assert f(target, drafts, m, V, x) == drafts + 4 * m * V
