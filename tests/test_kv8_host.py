"""Refusals of the paged 8-bit cache calls that the host makes before any launch, and the oracle's own checks (CPU)."""
import ctypes
import os

import numpy as np
import pytest

from .kv8_common import DECODE, GROUP, PAGE, Cache, Pages, attention, e4m3_encode, pow2_scale

FAKE = 1 << 20        # an aligned address that is never dereferenced: every check below fails first


@pytest.fixture(scope="module")
def lib():
    from paper_2609_06498_amd.runtime import library_path, load_library
    if not os.path.exists(library_path()):
        pytest.skip("libdflow.so not built")
    return load_library()


def kv8(**kw):
    from paper_2609_06498_amd.runtime import KV8
    a = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, num_pages=10, n_kv_heads=2, head_dim=128)
    a.update(kw)
    return KV8(*[a[n] for n, _ in KV8._fields_])


def pool(**kw):
    from paper_2609_06498_amd.runtime import Pool
    a = dict(page_table=FAKE, max_pages=4, n_held=FAKE, free_pages=FAKE, num_pages=10, n_free=FAKE)
    a.update(kw)
    return Pool(*[a[n] for n, _ in Pool._fields_])


BAD_CACHE = [(dict(k=None), -1), (dict(v=None), -1), (dict(k_scale=None), -1), (dict(v_scale=None), -1),
             (dict(k=FAKE + 8), -1), (dict(v_scale=FAKE + 2), -1), (dict(head_dim=96), -2), (dict(n_kv_heads=0), -2),
             (dict(num_pages=0), -4), (dict(num_pages=1 << 25), -4)]


@pytest.mark.parametrize("kw,code", BAD_CACHE)
def test_bad_cache_is_refused(lib, kw, code):
    c = ctypes.byref(kv8(**kw))
    assert lib.dflow_kv8_append(None, 1, c, 1, FAKE, 256, FAKE, 256, FAKE, FAKE) == code
    assert lib.dflow_kv8_attention(None, 1, c, 1, FAKE, 4, FAKE, FAKE, 1, 1, 64, 4, FAKE, 512, 0.1, 1, FAKE, 512, None, 0,
                                   FAKE) == code
    assert lib.dflow_last_error()


@pytest.mark.parametrize("at,value,code", [
    (1, 2, -3), (3, -1, -2), (4, None, -1), (4, FAKE + 2, -2), (5, 255, -2), (5, 260, -2), (6, None, -1), (7, 100, -2),
    (8, None, -1), (9, None, -1)])
def test_append_refusals(lib, at, value, code):
    args = [None, 1, ctypes.byref(kv8()), 1, FAKE, 256, FAKE, 256, FAKE, FAKE]
    args[at] = value
    assert lib.dflow_kv8_append(*args) == code


def test_no_rows_is_no_launch(lib):
    assert lib.dflow_kv8_append(None, 1, ctypes.byref(kv8()), 0, None, 0, None, 0, None, FAKE) == 0
    assert lib.dflow_kv8_attention(None, 1, ctypes.byref(kv8()), 1, FAKE, 4, FAKE, FAKE, 0, 0, 64, 4, None, 0, 0.1, 1,
                                   None, 0, None, 0, FAKE) == 0


@pytest.mark.parametrize("at,value,code", [
    (1, 5, -3), (3, 0, -4), (3, 70000, -4), (4, None, -1), (5, 0, -4), (6, None, -1), (7, None, -1), (8, -1, -2),
    (9, -1, -2), (9, 1 << 21, -2), (10, -1, -2), (11, 5, -2), (11, 0, -2), (12, None, -1), (12, FAKE + 4, -2),
    (13, 256, -2), (13, 513, -2), (14, 0.0, -1), (14, -1.0, -1), (14, float("nan"), -1), (14, float("inf"), -1),
    (16, None, -1), (17, 511, -2), (20, None, -1)])
def test_attention_refusals(lib, at, value, code):
    args = [None, 1, ctypes.byref(kv8()), 1, FAKE, 4, FAKE, FAKE, 1, 1, 64, 4, FAKE, 512, 0.1, 1, FAKE, 512, FAKE, 1 << 30,
            FAKE]
    args[at] = value
    assert lib.dflow_kv8_attention(*args) == code, lib.dflow_last_error()


@pytest.mark.parametrize("at,value,code", [(1, None, -1), (2, 0, -4), (2, 1025, -4), (3, None, -1), (4, None, -1),
                                           (6, -1, -2), (7, None, -1), (8, None, -1)])
def test_page_resize_refusals(lib, at, value, code):
    args = [None, ctypes.byref(pool()), 3, FAKE, FAKE, FAKE, 100, FAKE, FAKE]
    args[at] = value
    assert lib.dflow_page_resize(*args) == code


@pytest.mark.parametrize("kw,code", [(dict(page_table=None), -1), (dict(n_held=None), -1), (dict(free_pages=None), -1),
                                     (dict(n_free=None), -1), (dict(max_pages=0), -4), (dict(num_pages=0), -4),
                                     (dict(num_pages=1 << 26), -4), (dict(max_pages=1 << 26), -4)])
def test_bad_pool_is_refused(lib, kw, code):
    assert lib.dflow_page_resize(None, ctypes.byref(pool(**kw)), 3, FAKE, FAKE, FAKE, 100, FAKE, FAKE) == code


def test_workspace_refusals(lib):
    bad = ctypes.c_size_t(-1).value
    for args in ((7, 1, 1, 64, 4, 2, 128), (1, 0, 1, 64, 4, 2, 128), (1, 1, -1, 64, 4, 2, 128), (1, 1, 1, -1, 4, 2, 128),
                 (1, 1, 1, 64, 5, 2, 128), (1, 1, 1, 64, 4, 2, 80)):
        assert lib.dflow_kv8_attention_workspace(*args) == bad


def test_python_layer_needs_a_device():
    torch = pytest.importorskip("torch")
    from paper_2609_06498_amd import KV8Cache, PagePool
    from paper_2609_06498_amd.runtime import DFlowError
    z = torch.zeros(2, 1, PAGE, 64, dtype=torch.uint8)
    s = torch.ones(2, 1, 4)
    with pytest.raises(DFlowError, match="no CPU path"):
        KV8Cache(z, z.transpose(2, 3).contiguous(), s, s)
    i = lambda *n: torch.zeros(*n, dtype=torch.int32)
    with pytest.raises(DFlowError, match="no CPU path"):
        PagePool(i(2, 3), i(2), i(4), i(1))


# ---------------------------------------------------------------- the oracle
def test_oracle_codes_are_e4m3():
    """Against torch's own e4m3 type: every code's value, and the rounding of values between and at the middles."""
    torch = pytest.importorskip("torch")
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(DECODE, t)
    grid = np.unique(np.abs(DECODE[np.isfinite(DECODE)]))
    x = np.concatenate([grid, (grid[1:] + grid[:-1]) / 2, np.random.default_rng(0).uniform(-448, 448, 4000)])
    x = np.concatenate([x, -x]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(e4m3_encode(x), want)
    assert e4m3_encode(np.inf) == 126 and e4m3_encode(-1e9) == 254 and e4m3_encode(np.nan) == 127


def test_oracle_scale_and_append():
    assert pow2_scale(448.0) == 1.0 and pow2_scale(448.1) == 2.0 and pow2_scale(224.0) == 0.5 and pow2_scale(0) == 1.0
    assert pow2_scale(1e-45) == 2.0 ** -100
    rng = np.random.default_rng(1)
    c = Cache(2, 1, 64)
    x = rng.normal(0, 1, (20, 1, 64))
    c.append(x, x, np.arange(60, 80))
    rel = np.abs(c.values("k")[[0] * 4 + [1] * 16, 0, list(range(60, 64)) + list(range(16))] - x[:, 0])
    # half a step of e4m3 for normal codes, half the smallest step (2^-10 of the scale) below
    assert (rel <= np.maximum(2.0 ** -4 * np.abs(x[:, 0]), 2.0 ** -10 * c.scale["k"].max())).all()


def test_oracle_attention_against_torch():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(2)
    c = Cache(3, 2, 64)
    x, y = rng.normal(0, 1, (2, 100, 2, 64))
    t = np.array([[2, 0]])
    c.append(x, y, [t[0, p // PAGE] * PAGE + p % PAGE for p in range(100)])
    q = rng.normal(0, 1, (5, 4, 64))
    out, _, _ = attention(c, t, [100], [0, 5], q, True, 0.125)
    k, v = (torch.from_numpy(c.values(n)[t[0]].transpose(1, 0, 2, 3).reshape(2, 128, 64)[:, :100]) for n in "kv")
    k, v = k.repeat_interleave(2, 0), v.repeat_interleave(2, 0)
    mask = torch.arange(100)[None] <= torch.arange(95, 100)[:, None]
    want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q).transpose(0, 1)[None], k[None], v[None],
                                                            attn_mask=mask, scale=0.125)[0].transpose(0, 1)
    np.testing.assert_allclose(out, want.numpy(), rtol=1e-12, atol=1e-12)


def test_oracle_pages():
    p = Pages(np.full((3, 4), -1, np.int32), [0] * 3, [9, 8, 7, 6, 5])
    slots, starts, ok = p.resize([0, 0, 0], [70, 1, 0])
    assert ok and p.table[0].tolist() == [5, 6, -1, -1] and p.table[1, 0] == 7 and p.free == [9, 8]
    assert slots[:2] == [5 * PAGE, 5 * PAGE + 1] and slots[64] == 6 * PAGE and slots[70] == 7 * PAGE
    assert starts.tolist() == [0, 70, 71, 71]
    assert not p.resize([70, 1, 0], [0, 64 * 3, 1])[2] and p.held == [2, 1, 0]     # the second asks for too much
    assert p.resize([0, 1, 0], None)[2] and p.free == [9, 8, 6, 5]
    assert GROUP == 16
