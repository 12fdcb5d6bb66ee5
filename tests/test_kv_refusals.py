"""What the calls of the key-value cache refuse, and the frequencies of the rotation: host code, no GPU needed."""
import ctypes as C
import os

import numpy as np
import pytest

from oracle import kv_oracle as O


@pytest.fixture(scope="module")
def b():
    from paper_2312_11514_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2312_11514_amd.build import build_library
        build_library()
    binding.load_library()
    return binding


GOOD = dict(layers=2, heads=8, kv_heads=2, head_dim=64, page_tokens=16, pages=100, max_seqs=4, max_pages=20, max_tokens=5, dtype=1, norm=1,
            rotary=0, rotary_dim=32, norm_eps=1e-5, rotary_scale=1.0, scale=0.125)


def _config(b, **changes):
    cfg = b.LifKvConfig()
    for k, v in dict(GOOD, **changes).items():
        setattr(cfg, k, v)
    return cfg


def _buffers(b, cfg, **changes):
    p = 1 << 32
    buf = b.LifKvBuffers(p, p, p, p, p, p, p, p, b.load_library().lif_kv_workspace_bytes(C.byref(cfg)))
    for k, v in changes.items():
        setattr(buf, k, v)
    return buf


def _create(b, cfg, buf):
    h = C.c_void_p()
    return b.load_library().lif_kv_create(C.byref(cfg), C.byref(buf), C.byref(h)), h


@pytest.mark.parametrize("change", [
    dict(layers=0), dict(heads=7), dict(heads=0), dict(kv_heads=0), dict(kv_heads=16), dict(head_dim=0), dict(head_dim=60), dict(head_dim=264),
    dict(page_tokens=8), dict(page_tokens=24), dict(page_tokens=512), dict(page_tokens=0), dict(page_tokens=-16), dict(pages=0),
    dict(pages=(1 << 24) + 1), dict(max_seqs=0), dict(max_seqs=1025), dict(max_pages=0), dict(max_pages=(1 << 20) + 1),
    dict(max_pages=1 << 20, page_tokens=32), dict(max_tokens=0), dict(max_tokens=257), dict(dtype=3), dict(dtype=-1), dict(norm=3), dict(rotary=2),
    dict(rotary_dim=-2), dict(rotary_dim=66), dict(rotary_dim=24), dict(rotary_dim=3, rotary=1), dict(norm_eps=-1.0),
    dict(norm_eps=float("nan")), dict(scale=float("inf")), dict(scale=float("nan")), dict(rotary_scale=float("nan"))])
def test_configurations(b, change):
    cfg = _config(b, **change)
    assert b.load_library().lif_kv_workspace_bytes(C.byref(cfg)) == 0
    buf = _buffers(b, _config(b))
    assert _create(b, cfg, buf)[0] == b.LIF_INVALID_ARG


def test_buffers(b):
    cfg = _config(b)
    assert b.load_library().lif_kv_workspace_bytes(C.byref(cfg)) % 256 == 0
    for name in ("k", "v", "table", "lengths", "fresh", "refs", "workspace", "frequencies"):
        assert _create(b, cfg, _buffers(b, cfg, **{name: None}))[0] == b.LIF_INVALID_ARG, name
    for change in (dict(k=(1 << 32) + 8), dict(v=(1 << 32) + 2), dict(workspace=(1 << 32) + 128), dict(workspace_bytes=256)):
        assert _create(b, cfg, _buffers(b, cfg, **change))[0] == b.LIF_INVALID_ARG, change
    plain = _config(b, rotary_dim=0)
    rc, h = _create(b, plain, _buffers(b, plain, frequencies=None))
    assert rc == b.LIF_OK and b.load_library().lif_kv_destroy(h) == b.LIF_OK
    assert b.load_library().lif_kv_destroy(None) == b.LIF_OK
    assert b.load_library().lif_kv_create(None, None, None) == b.LIF_INVALID_ARG
    assert b.load_library().lif_kv_workspace_bytes(None) == 0


def test_calls(b):
    lib, cfg, p = b.load_library(), _config(b), 1 << 32
    rc, h = _create(b, cfg, _buffers(b, cfg))
    assert rc == b.LIF_OK
    bad = b.LIF_INVALID_ARG
    assert lib.lif_kv_reset(None, None) == lib.lif_kv_adopt(None, None) == lib.lif_kv_compact(None, None) == bad
    assert lib.lif_kv_reserve(h, None, None) == lib.lif_kv_reserve(None, p, None) == bad
    assert lib.lif_kv_truncate(h, None, None) == lib.lif_kv_truncate(None, p, None) == bad
    for src, dst, n in ((None, p, 1), (p, None, 1), (p, p, 0), (p, p, -1), (p, p, 5)):
        assert lib.lif_kv_fork(h, src, dst, n, None) == bad
    assert lib.lif_kv_get_state(h, None, None) == lib.lif_kv_get_state(None, C.byref(b.LifKvState()), None) == bad
    rows = dict(q=p, k=p, v=p, q_out=p, q_stride=512, k_stride=128, v_stride=128, q_out_stride=512, batch=2, n_tokens=5)
    for layer, change in ((-1, {}), (2, {}), (0, dict(batch=0)), (0, dict(batch=1025)), (0, dict(n_tokens=0)), (0, dict(n_tokens=6)), (0, dict(q=None)),
                          (0, dict(k=None)), (0, dict(v=None)), (0, dict(q_out=None)), (0, dict(q=p + 8)), (0, dict(k=p + 2)), (0, dict(v=p + 4)),
                          (0, dict(q_out=p + 8)), (0, dict(q_stride=504)), (0, dict(q_stride=516)), (0, dict(k_stride=120)),
                          (0, dict(v_stride=130)), (0, dict(q_out_stride=-512)), (0, dict(q_out_stride=1 << 41))):
        assert lib.lif_kv_append(h, layer, C.byref(b.LifKvRows(**dict(rows, **change))), None) == bad, (layer, change)
    query = dict(q=p, out=p, q_stride=512, out_stride=512, batch=2, n_tokens=5)
    for layer, change in ((-1, {}), (2, {}), (0, dict(batch=0)), (0, dict(n_tokens=6)), (0, dict(q=None)), (0, dict(out=None)), (0, dict(q=p + 8)),
                          (0, dict(out=p + 8)), (0, dict(q_stride=8)), (0, dict(out_stride=513)), (0, dict(window=-1))):
        assert lib.lif_kv_attend(h, layer, C.byref(b.LifKvQuery(**dict(query, **change))), None) == bad, (layer, change)
    assert lib.lif_kv_append(h, 0, None, None) == lib.lif_kv_attend(h, 0, None, None) == bad
    wide = _config(b, max_tokens=65)
    rc, w = _create(b, wide, _buffers(b, wide))
    assert lib.lif_kv_attend(w, 0, C.byref(b.LifKvQuery(**dict(query, n_tokens=65, tree=p))), None) == bad
    assert b"64" in lib.lif_last_error_string()
    lib.lif_kv_destroy(h)
    lib.lif_kv_destroy(w)


@pytest.mark.parametrize("dim,base", [(2, 10000.0), (16, 10000.0), (32, 500.0), (128, 1e6), (80, 10000.0)])
@pytest.mark.parametrize("kind,args", [("plain", {}), ("linear", dict(factor=4.0)), ("base", dict(factor=2.5)), ("ramp", dict(factor=8.0, trained=2048)),
                                       ("ramp", dict(factor=8.0, trained=8192, slow=1.0, fast=4.0))])
def test_frequencies(b, dim, base, kind, args):
    import paper_2312_11514_amd as lif
    kinds = {"plain": lif.ROPE_PLAIN, "linear": lif.ROPE_LINEAR, "base": lif.ROPE_BASE, "ramp": lif.ROPE_RAMP}
    if kind == "base" and dim == 2:
        with pytest.raises(lif.LifError):
            lif.rope_frequencies(dim, base, kinds[kind], **args)
        return
    got = lif.rope_frequencies(dim, base, kinds[kind], **args).numpy()
    np.testing.assert_allclose(got, O.frequencies(dim, base, kind, **args), rtol=1e-13)
    if kind == "base":                                     # the fastest pair as before, the slowest `factor` times slower
        plain = O.frequencies(dim, base)
        assert got[0] == plain[0] and abs(got[-1] * args["factor"] / plain[-1] - 1) < 1e-12


@pytest.mark.parametrize("dim,args", [(0, {}), (3, {}), (-2, {}), (4, dict(base=0.0)), (4, dict(base=float("inf"))), (4, dict(scaling=4)),
                                      (4, dict(scaling=1, factor=0.0)), (4, dict(scaling=3, factor=2.0)),
                                      (4, dict(scaling=3, factor=2.0, trained=10.0, slow=4.0, fast=4.0))])
def test_frequencies_refused(b, dim, args):
    import paper_2312_11514_amd as lif
    with pytest.raises(lif.LifError):
        lif.rope_frequencies(dim, **args)


# ---- the oracle against what it has to be by hand -------------------------------------------------------------------------------

def test_oracle_attention_by_hand():
    q, k, v = np.array([[[1.0, 0.0]]]), np.array([[[0.0, 5.0], [np.log(3.0), 2.0]]]), np.array([[[4.0, 0.0], [0.0, 8.0]]])
    out, lse, _, _ = O.attend(q, k, v, np.ones((1, 2), bool), 1.0)
    np.testing.assert_allclose(out, [[[1.0, 6.0]]])
    np.testing.assert_allclose(lse, [[np.log(4.0)]])
    out, lse, _, _ = O.attend(q, k, v, np.zeros((1, 2), bool), 1.0)
    assert (out == 0).all() and np.isneginf(lse).all()


def test_oracle_rotation_turns_inner_products_by_the_distance():
    f = O.frequencies(8)
    rng = np.random.default_rng(0)
    x, y = rng.standard_normal((2, 1, 8))
    for layout in ("half", "interleaved"):
        at = lambda i, j: float((O.rotate(x, i, f, layout) * O.rotate(y, j, f, layout)).sum())
        assert abs(at(7, 3) - at(104, 100)) < 1e-12 and abs(at(7, 3) - at(3, 7)) > 1e-6


def test_oracle_visible():
    assert O.visible(4, 2).tolist() == [[True, True, True, False], [True, True, True, True]]
    assert O.visible(4, 2, start=1, window=2).tolist() == [[False, True, True, False], [False, False, True, True]]
    assert O.visible(3, 2, tree=[1, 2]).tolist() == [[True, True, False], [True, False, True]]


def test_oracle_pages():
    o = O.PagedOracle(6, 3, 4, 16)
    o.reserve([20, 16, 0])
    assert o.tables == [[0, 1], [2], []]
    o.fork([0], [2])
    assert o.tables[2] == [0, 3] and o.content[3] == ("initial", 1) and o.refs() == [2, 1, 1, 1, 0, 0]
    o.truncate([0, 0, -1])
    o.compact()
    assert o.tables == [[], [], [0, 1]] and o.content[1] == ("initial", 1) and o.used() == 2


@pytest.mark.parametrize("scale", [0.0, -0.125])
def test_scales_that_are_not_positive(b, scale):
    cfg = _config(b, scale=scale)
    assert b.load_library().lif_kv_workspace_bytes(C.byref(cfg)) == 0


def test_the_hint(b):
    lib, cfg = b.load_library(), _config(b)
    rc, h = _create(b, cfg, _buffers(b, cfg))
    assert rc == b.LIF_OK
    assert lib.lif_kv_set_expected_tokens(None, 5) == lib.lif_kv_set_expected_tokens(h, -1) == b.LIF_INVALID_ARG
    assert lib.lif_kv_set_expected_tokens(h, 0) == lib.lif_kv_set_expected_tokens(h, 1 << 30) == b.LIF_OK
    lib.lif_kv_destroy(h)


def test_a_page_of_two_gib(b):
    assert b.load_library().lif_kv_workspace_bytes(C.byref(_config(b, heads=65536, kv_heads=65536, head_dim=256, page_tokens=256, dtype=0))) == 0


def test_too_many_steps(b):
    """1024 sequences of 2^24 positions, 64 key heads: more steps than 32 bits count"""
    lib = b.load_library()
    cfg = _config(b, heads=64, kv_heads=64, max_seqs=1024, max_pages=1 << 20)
    rc, h = _create(b, cfg, _buffers(b, cfg))
    assert rc == b.LIF_OK
    p = 1 << 32
    query = b.LifKvQuery(q=p, out=p, q_stride=4096, out_stride=4096, batch=1024, n_tokens=1)
    assert lib.lif_kv_attend(h, 0, C.byref(query), None) == b.LIF_INVALID_ARG and b"together" in lib.lif_last_error_string()
    lib.lif_kv_destroy(h)
