"""Arrays of a matrix that share memory are refused: host code, no GPU needed."""
import ctypes as C

import pytest

from tests.test_packed_refusals import CONFIG, P, _refused, b  # noqa: F401


@pytest.mark.parametrize("codes,groups,shared", [(0, 0, True), (0, 112 * 384 // 2 - 16, True), (112 * 6 * 4 - 16, 0, True), (16, 0, True),
                                                 (0, 112 * 384 // 2, False), (112 * 6 * 4, 0, False)])
def test_codes_and_groups_lie_beside_each_other(b, codes, groups, shared):  # noqa: F811
    lib, h, cfg = b.load_library(), C.c_void_p(), b.LifPackedConfig(**CONFIG)
    sizes = lib.lif_packed_code_bytes(C.byref(cfg)), lib.lif_packed_group_bytes(C.byref(cfg))
    assert sizes == (112 * 384 // 2, 112 * 6 * 4)
    # (more bytes than needed are no part of the matrix)
    buf = b.LifPackedBuffers(P + codes, P + groups, sizes[0] + 4096, sizes[1] + 4096)
    rc = lib.lif_packed_create(C.byref(cfg), C.byref(buf), C.byref(h))
    if shared:
        _refused(b, rc, "overlap")
    else:
        assert rc == 0 and lib.lif_packed_destroy(h) == 0
