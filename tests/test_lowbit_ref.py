"""The references of the 8-bit cache and the 4-bit weights against torch's own types and against themselves (CPU), and the
refusals of their entry points, none of which reaches the GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import lowbit_ref as lr
from paper_2608_15943_amd import binding as kb


def test_e4m3_codes_are_those_of_the_type():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(lr.E4M3, want, equal_nan=True)
    x = np.random.default_rng(1).uniform(-448, 448, 20000) * 2.0 ** np.random.default_rng(2).integers(-20, 1, 20000)
    x[:252] = np.concatenate([(lr._POS[1:] + lr._POS[:-1]) / 2, -(lr._POS[1:] + lr._POS[:-1]) / 2])     # ties
    got = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(lr.e4m3(x.astype(np.float32).astype(np.float64)), got)


@pytest.mark.parametrize("m,s", [(448.0, 1.0), (448.001, 2.0), (224.0, 0.5), (1.0, 2.0**-8), (1.75, 2.0**-8),
                                 (1.76, 2.0**-7), (0.0, 2.0**-100), (1e-40, 2.0**-100), (np.inf, np.nan)])
def test_scale_is_the_least_power_of_two(m, s):
    assert lr.scale_of(m) == s or (np.isnan(s) and np.isnan(lr.scale_of(m)))


def test_written_cache_reads_back_within_half_a_step():
    rng = np.random.default_rng(3)
    kv = rng.standard_normal((2, 70, 2, lr.D))
    c = lr.Cache(2, 5)
    c.write([[3, 1]], 0, kv)
    got = c.values([[3, 1]], 0, 70)
    for j in range(0, 70, lr.BLK):
        x, y = kv[:, j: j + lr.BLK], got[:, j: j + lr.BLK]
        s = np.abs(x).max((1, 3), keepdims=True) / 224        # the scale is below twice the least that fits
        assert (np.abs(x - y) <= np.maximum(2.0**-4 * np.abs(x), 2.0**-10 * s)).all()


@pytest.mark.parametrize("N,K,group", [(5, 128, 32), (33, 256, 64), (16, 384, 128)])
def test_packed_weights_layout(N, K, group):
    """Every code and scale is where the header says, read back one by one."""
    rng = np.random.default_rng(N)
    codes, s = lr.w4_codes(lr.bf16(rng.standard_normal((N, K)).astype(np.float32)), group)
    buf = lr.w4_pack(codes, s)
    assert buf.size == kb.kvp_w4_bytes(N, K, group)
    nb = (N + 15) // 16
    words = buf[: nb * 8 * K].view(np.uint32)
    scales = buf[nb * 8 * K:].view(np.uint16)
    for n, k in zip(rng.integers(0, N, 200), rng.integers(0, K, 200)):
        w, j, e = k % 128 // 32, k % 32 // 8, k % 8
        word = words[((n // 16 * (K // 128) + k // 128) * 64 + 16 * j + n % 16) * 4 + w]
        assert (int(word) >> (4 * (e // 2) + 16 * (e % 2))) & 15 == codes[n, k]
        sb = scales[(n // 16 * (K // group) + k // group) * 16 + n % 16]
        assert np.array([int(sb) << 16], np.uint32).view(np.float32)[0] == s[n, k // group]


# ---- refusals -----------------------------------------------------------------------------------

P = 4096          # a non-null, aligned address that no refused call reads


def _model(L=2, a=4, g=2, dtype=kb.KVP_DTYPE_BF16, tau=(0, 0), max_batch=4, max_seq=256):
    return kb.Model(L, a * 128, a, g, 128, dtype, list(tau), max_batch=max_batch, max_seq=max_seq, kv_capacity=max_seq)


def _rows(**kw):
    d = dict(cu=P, len=P, pages=P, pages_stride=4, B=2, rows=6, max_new=4, max_pos=200)
    d.update(kw)
    return kb.kvp_rows(**d)


def _code(f, *a):
    with pytest.raises(kb.KvpError) as e:
        f(*a)
    return e.value.code


def test_pool_refusals():
    m = _model()
    for args in ((0, 0, P, P, 3), (0, P, 0, P, 3), (0, P, P, 0, 3), (0, P, P, P, 0), (1, P, P, P, 3), (2, P, P, P, 3),
                 (-1, P, P, P, 3), (0, P + 8, P, P, 3), (0, P, P + 1, P, 3), (0, P, P, P + 4, 3)):
        assert _code(m.kvp_set_kv_pool_fp8, *args) == kb.KVP_E_INVALID_ARG, args
    f = kb.Model(1, 128, 1, 1, 128, kb.KVP_DTYPE_FP32, [0], max_batch=1, max_seq=4, kv_capacity=4)
    assert _code(f.kvp_set_kv_pool_fp8, 0, P, P, P, 3) == kb.KVP_E_SHAPE
    assert _code(f.kvp_page_bytes_fp8) == kb.KVP_E_SHAPE
    assert _code(f.kvp_workspace_size, kb.KVP_PHASE_STEP_FP8, 1, 1) == kb.KVP_E_SHAPE
    assert _code(f.kvp_append_fp8, 0, P, P, P, 128, _rows(), P) == kb.KVP_E_SHAPE
    assert m.kvp_page_bytes_fp8() == 2 * (2 * 64 * 128 + 32)


ROWS = [(dict(len=0), kb.KVP_E_INVALID_ARG), (dict(pages=0), kb.KVP_E_INVALID_ARG),
        (dict(pages_stride=0), kb.KVP_E_INVALID_ARG), (dict(pages_stride=1 << 30), kb.KVP_E_INVALID_ARG),
        (dict(B=0), kb.KVP_E_INVALID_ARG), (dict(rows=0), kb.KVP_E_INVALID_ARG), (dict(max_new=0), kb.KVP_E_INVALID_ARG),
        (dict(max_pos=-1), kb.KVP_E_INVALID_ARG), (dict(cu=0), kb.KVP_E_INVALID_ARG),
        (dict(cu=0, rows=2, max_new=2), kb.KVP_E_INVALID_ARG), (dict(B=5), kb.KVP_E_CAPACITY),
        (dict(max_new=257), kb.KVP_E_CAPACITY), (dict(rows=4 * 256 + 1), kb.KVP_E_CAPACITY),
        (dict(max_pos=256), kb.KVP_E_CAPACITY), (dict(max_pos=2**31 - 1), kb.KVP_E_CAPACITY)]


@pytest.mark.parametrize("kw,code", ROWS)
def test_row_refusals(kw, code):
    m = _model()
    m.kvp_set_kv_pool_fp8(0, P, P, P, 3)
    r = _rows(**kw)
    assert _code(m.kvp_append_fp8, 0, P, P, P, 1024, r, P + 16) == code
    assert _code(m.kvp_attention_fp8, 0, P, r, P + 16, P, 1 << 40) == code
    assert _code(m.kvp_step_fp8, P, r, P + 16, P, 1 << 40) == code


def test_append_refusals():
    m, r = _model(), _rows()
    assert _code(m.kvp_append_fp8, 0, P, P, P, 1024, r, P) == kb.KVP_E_STATE        # no pools yet
    m.kvp_set_kv_pool_fp8(0, P, P, P, 3)
    for args in ((2, P, P, P, 1024, r, P + 16), (-1, P, P, P, 1024, r, P + 16), (0, P, P, P, 1024, r, 0), (0, 0, P, P, 1024, r, P),
                 (0, P, P, 0, 1024, r, P + 16), (0, P, 0, P, 1024, r, P + 16), (0, 0, 0, 0, 1024, r, 0),
                 (1, P, P, P, 1024, r, P + 16), (0, P, P, P, 1020, r, P + 16), (0, P, P, P, 504, r, P + 16),
                 (0, 0, P, P, 248, r, 0), (0, P + 2, P, P, 1024, r, P + 16), (0, P, P + 2, P, 1024, r, P + 16),
                 (0, P, P, P + 2, 1024, r, P + 16), (0, P, P, P, 1024, r, P + 2), (0, P, P, P, 1024, r, P)):
        assert _code(m.kvp_append_fp8, *args) == kb.KVP_E_INVALID_ARG, args
    assert kb.lib().kvp_append_fp8(None, 0, P, P, P, 1024, C.byref(r), P, None) == kb.KVP_E_INVALID_ARG
    assert kb.lib().kvp_append_fp8(m.ctx, 0, P, P, P, 1024, None, P, None) == kb.KVP_E_INVALID_ARG


def test_attention_and_step_refusals():
    m, r = _model(), _rows()
    n = m.kvp_workspace_size(kb.KVP_PHASE_STEP_FP8, 2, 6)
    assert _code(m.kvp_attention_fp8, 0, P, r, P + 16, P, n) == kb.KVP_E_STATE
    assert _code(m.kvp_step_fp8, P, r, P + 16, P, n) == kb.KVP_E_STATE
    m.kvp_set_kv_pool_fp8(0, P, P, P, 3)
    assert _code(m.kvp_step_fp8, P, r, P + 16, P, n) == kb.KVP_E_STATE                # no weights
    for args in ((0, 0, r, P), (0, P, r, 0), (0, P, r, P), (0, P + 2, r, P + 16), (0, P, r, P + 2), (2, P, r, P + 16)):
        assert _code(m.kvp_attention_fp8, *args, P, n) == kb.KVP_E_INVALID_ARG, args
    for args in ((0, r, P), (P, r, 0), (P, r, P), (P + 2, r, P + 16), (P, r, P + 2)):
        assert _code(m.kvp_step_fp8, *args, P, n) == kb.KVP_E_INVALID_ARG, args
    for ws, k in ((0, n), (P, n - 1), (P + 8, n)):
        assert _code(m.kvp_attention_fp8, 0, P, r, P + 16, ws, k) == kb.KVP_E_WORKSPACE
        assert _code(m.kvp_step_fp8, P, r, P + 16, ws, k) == kb.KVP_E_WORKSPACE
    assert _code(m.kvp_workspace_size, kb.KVP_PHASE_STEP_FP8, 5, 6) == kb.KVP_E_CAPACITY
    assert _code(m.kvp_workspace_size, kb.KVP_PHASE_STEP_FP8, 4, 1025) == kb.KVP_E_CAPACITY
    assert _code(m.kvp_workspace_size, kb.KVP_PHASE_STEP_FP8, 4, 0) == kb.KVP_E_INVALID_ARG


def test_step_workspace_never_shrinks():
    m = _model(L=1, a=32, g=8, tau=(0,), max_batch=64, max_seq=4096)
    last = 0
    for B, rows in ((1, 1), (1, 2), (2, 16), (2, 63), (4, 64), (4, 65), (4, 66), (8, 200), (64, 2000), (64, 64 * 4096)):
        n = m.kvp_workspace_size(kb.KVP_PHASE_STEP_FP8, B, rows)
        assert n >= last, (B, rows)
        last = n


def test_w4_refusals():
    assert kb.kvp_w4_bytes(17, 256, 64) == 2 * (16 * 128 + 16 * 4 * 2)
    for K, g in ((64, 32), (200, 32), (0, 32), (128, 16), (128, 0), (256, 256), (-128, 32)):
        assert _code(kb.kvp_w4_bytes, 16, K, g) == kb.KVP_E_SHAPE
        assert _code(kb.kvp_pack_w4, P, 16, K, g, P) == kb.KVP_E_SHAPE
        assert _code(kb.kvp_linear_w4, P, P, 0, P + 16, 1, 16, K, g) == kb.KVP_E_SHAPE
    assert _code(kb.kvp_w4_bytes, 0, 128, 32) == kb.KVP_E_INVALID_ARG
    for args in ((0, 16, 128, 32, P), (P, 16, 128, 32, 0), (P, 0, 128, 32, P), (P + 2, 16, 128, 32, P), (P, 16, 128, 32, P + 2)):
        assert _code(kb.kvp_pack_w4, *args) == kb.KVP_E_INVALID_ARG, args
    assert _code(kb.kvp_pack_w4, P, (1 << 20) + 1, 128, 32, P) == kb.KVP_E_SHAPE
    assert _code(kb.kvp_w4_bytes, 16, (1 << 20) + 128, 32) == kb.KVP_E_SHAPE
    assert _code(kb.kvp_pack_w4, P, 16, (1 << 20) + 128, 32, P) == kb.KVP_E_SHAPE
    assert _code(kb.kvp_linear_w4, P, P, 0, P + 16, 1, 16, (1 << 20) + 128, 32) == kb.KVP_E_SHAPE
    for x, w, res, y, M, N in ((0, P, 0, P, 1, 16), (P, 0, 0, P + 16, 1, 16), (P, P, 0, 0, 1, 16), (P, P, 0, P + 16, 0, 16),
                               (P, P, 0, P + 16, 1, 0), (P, P, 0, P, 1, 16), (P + 2, P, 0, P, 1, 16), (P, P + 2, 0, P + 16, 1, 16),
                               (P, P, P + 2, P + 16, 1, 16), (P, P, 0, P + 2, 1, 16)):
        assert _code(kb.kvp_linear_w4, x, w, res, y, M, N, 128, 32) == kb.KVP_E_INVALID_ARG, (x, w, res, y, M, N)
    for M, N in (((1 << 20) + 1, 16), (1, (1 << 20) + 1)):
        assert _code(kb.kvp_linear_w4, P, P, 0, P + 16, M, N, 128, 32) == kb.KVP_E_SHAPE


def test_set_layer_w4_refusals():
    m = _model()
    for args in ((0, 0, P, P, P, 32), (0, P, 0, P, P, 32), (0, P, P, 0, P, 32), (0, P, P, P, 0, 32), (1, P, P, P, P, 32),
                 (1, P, 0, P, P, 32), (2, P, P, P, P, 32), (-1, P, P, P, P, 32), (0, P + 2, P, P, P, 32), (0, P, P, P, P + 2, 32),
                 (0, 0, 0, 0, 0, 32)):
        assert _code(m.kvp_set_layer_w4, *args) == kb.KVP_E_INVALID_ARG, args
    assert _code(m.kvp_set_layer_w4, 0, P, P, P, P, 16) == kb.KVP_E_SHAPE
    f = kb.Model(1, 128, 1, 1, 128, kb.KVP_DTYPE_FP32, [0], max_batch=1, max_seq=4, kv_capacity=4)
    assert _code(f.kvp_set_layer_w4, 0, P, P, P, P, 32) == kb.KVP_E_SHAPE
    # Without bf16 weights the prefill has none, the steps have.
    m.kvp_set_layer_w4(0, P, P, P, P, 32)
    m.kvp_set_layer_w4(1, P, 0, 0, P, 32)
    m.kvp_set_kv_slot(0, P, P)
    n = m.kvp_workspace_size(kb.KVP_PHASE_PREFILL, 1, 8)
    assert _code(m.kvp_prefill, P, P + 16, 1, 8, P, n) == kb.KVP_E_STATE
    m.kvp_set_layer_w4(1, 0, 0, 0, 0, 0)
    n = m.kvp_workspace_size(kb.KVP_PHASE_DECODE, 1)
    assert _code(m.kvp_decode_step, P, P, 3, P + 16, 1, P, n) == kb.KVP_E_STATE       # layer 1 has none again
