"""4-bit weights on the GPU: kvp_pack_w4 and kvp_linear_w4 against 64-bit references, and decode steps on them."""
import numpy as np
import pytest
import torch

import kvp_inputs as ki
import lowbit_ref as lr
from gpu_util import build_device_model, oracle_weights, rel_err, say, small_workload, to_np, workspace
from kvp_inputs import device as kd
from oracle import attention as oat
from paper_2608_15943_amd import binding as kb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kb.lib()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).cuda()


def _normal(rng, *shape):
    return lr.bf16(rng.standard_normal(shape).astype(np.float32))


def _packed(w, group):
    N, K = w.shape
    buf = torch.full((kb.kvp_w4_bytes(N, K, group) + 64,), 0xAB, dtype=torch.uint8, device="cuda")
    t = _dev(w)
    kb.kvp_pack_w4(t.data_ptr(), N, K, group, buf.data_ptr(), _stream())
    torch.cuda.synchronize()
    assert (buf[-64:] == 0xAB).all()          # nothing behind the buffer
    return buf[:-64]


@pytest.mark.parametrize("N,K,group", [(16, 128, 128), (1, 128, 32), (37, 256, 64), (100, 640, 128), (513, 1024, 32)])
def test_pack(N, K, group):
    rng = np.random.default_rng(N)
    w = _normal(rng, N, K) * np.float32(0.05)
    w = lr.bf16(w)
    w[0, :group] = 0                                  # a group of zeros
    w[N // 2, :5] = [1e-40, -1e-39, 0, 0, 0]          # its scale may vanish
    w[N // 2, 5:group] = 0
    codes, s = lr.w4_codes(w, group)
    assert np.array_equal(_packed(w, group).cpu().numpy(), lr.w4_pack(codes, s))


@pytest.mark.parametrize("N,K", [((1 << 20), 128), ((1 << 20) - 16, 128), (1, 1 << 20)])
def test_pack_and_linear_of_the_largest_sizes(N, K):
    """The first and last outputs of the longest matrices; the rest repeats 16 outputs."""
    rng = np.random.default_rng(8)
    w = lr.bf16(_normal(rng, min(N, 16), K) * np.float32(0.05))
    codes, s = lr.w4_codes(w, 128)
    t = _dev(w).repeat(max(N // 16, 1), 1)
    n = kb.kvp_w4_bytes(N, K, 128)
    buf = torch.full((n + 64,), 0xAB, dtype=torch.uint8, device="cuda")
    kb.kvp_pack_w4(t.data_ptr(), N, K, 128, buf.data_ptr(), _stream())
    torch.cuda.synchronize()
    assert (buf[-64:] == 0xAB).all()
    one = torch.from_numpy(lr.w4_pack(codes, s)).cuda()
    nb, cb = (N + 15) // 16, 8 * K          # blocks, bytes of one's codes
    assert torch.equal(buf[: nb * cb].view(nb, cb), one[:cb].expand(nb, cb))
    assert torch.equal(buf[nb * cb: n].view(nb, K // 4), one[cb:].expand(nb, K // 4))
    x = _normal(rng, 3, K)
    got = _linear(x, buf[:n], N, 128)
    y = x.astype(np.float64) @ lr.w4_weights(codes, s, 128).T
    tol = lr.linear_bound(x.astype(np.float64), y, s, 128)
    assert (np.abs(got.reshape(3, -1, min(N, 16)) - y[:, None]) <= tol[:, None]).all()


def test_pack_not_finite():
    w = _normal(np.random.default_rng(1), 20, 256)
    w[3, 100], w[4, 7], w[5, 255] = np.nan, np.inf, -np.inf
    got = _packed(w, 64).cpu().numpy()
    sb = (got[2 * 8 * 256:].view(np.uint16).astype(np.uint32) << 16).view(np.float32).reshape(2, 4, 16).transpose(0, 2, 1).reshape(32, 4)
    bad = np.zeros((32, 4), bool)
    bad[3, 1] = bad[4, 0] = bad[5, 3] = True
    assert np.array_equal(np.isnan(sb), bad)


def _linear(x, buf, N, group, res=None, inplace=False):
    M, K = x.shape
    dx = _dev(x)
    dr = None if res is None else _dev(res)
    y = dr if inplace else torch.full((M * N + 64,), 33.0, dtype=torch.bfloat16, device="cuda")
    kb.kvp_linear_w4(dx.data_ptr(), buf.data_ptr(), 0 if dr is None else dr.data_ptr(), y.data_ptr(), M, N, K, group, _stream())
    torch.cuda.synchronize()
    if not inplace:
        assert (y[M * N:] == 33.0).all()
    return y[: M * N].float().cpu().numpy().reshape(M, N) if not inplace else y.float().cpu().numpy()


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 33, 48, 49, 64, 65, 130])
@pytest.mark.parametrize("N,K,group", [(16, 128, 128), (40, 384, 32), (101, 1152, 64), (512, 4096, 128), (33, 2048, 32)])
def test_linear(M, N, K, group):
    rng = np.random.default_rng(M + N)
    codes, s = lr.w4_codes(_normal(rng, N, K), group)
    buf = torch.from_numpy(lr.w4_pack(codes, s)).cuda()
    x = _normal(rng, M, K) + lr.bf16(np.float32(0.5))      # a mean, which the codes' offset meets
    x = lr.bf16(x)
    y = x.astype(np.float64) @ lr.w4_weights(codes, s, group).T
    got = _linear(x, buf, N, group)
    tol = lr.linear_bound(x.astype(np.float64), y, s, group)
    assert (np.abs(got - y) <= tol).all(), np.abs((got - y) / tol).max()


@pytest.mark.parametrize("M", [3, 16, 32, 64, 200])
@pytest.mark.parametrize("N,K,group", [(4100, 256, 32), (8195, 128, 64), (12288, 1280, 128), (17000, 256, 128)])
def test_linear_many_outputs(M, N, K, group):
    """One to four blocks of 16 outputs a workgroup, with blocks left over."""
    say(f"[linear w4] M={M} N={N} K={K} group={group}")
    rng = np.random.default_rng(M + N)
    codes, s = lr.w4_codes(lr.bf16(_normal(rng, N, K) * np.float32(0.1)), group)
    buf = torch.from_numpy(lr.w4_pack(codes, s)).cuda()
    x = _normal(rng, M, K)
    y = x.astype(np.float64) @ lr.w4_weights(codes, s, group).T
    got = _linear(x, buf, N, group)
    assert (np.abs(got - y) <= lr.linear_bound(x.astype(np.float64), y, s, group)).all()


@pytest.mark.parametrize("inplace", [False, True])
def test_linear_residual(inplace):
    rng = np.random.default_rng(3)
    codes, s = lr.w4_codes(_normal(rng, 272, 512), 64)
    buf = torch.from_numpy(lr.w4_pack(codes, s)).cuda()
    x, res = _normal(rng, 5, 512), _normal(rng, 5, 272)
    y = x.astype(np.float64) @ lr.w4_weights(codes, s, 64).T + res
    got = _linear(x, buf, 272, 64, res, inplace)
    assert (np.abs(got - y) <= lr.linear_bound(x.astype(np.float64), y, s, 64)).all()


def test_linear_every_code_and_scale():
    """One input at a time: every code's value times its scale, exactly what the definition says (rounded to bf16 once)."""
    K, N, group = 128, 16, 32
    codes = (np.arange(N)[:, None] + np.arange(K)[None]) % 16
    s = lr.bf16(2.0 ** np.arange(-32, 32).reshape(N, 4).astype(np.float32) * np.float32(1.375))
    buf = torch.from_numpy(lr.w4_pack(codes, s)).cuda()
    x = np.eye(K, dtype=np.float32)
    got = _linear(x, buf, N, group)
    assert np.array_equal(got, lr.bf16(lr.w4_weights(codes, s, group).T.astype(np.float32)))


def test_linear_rows_that_are_not_finite_stay_apart():
    rng = np.random.default_rng(5)
    codes, s = lr.w4_codes(_normal(rng, 64, 512), 128)
    buf = torch.from_numpy(lr.w4_pack(codes, s)).cuda()
    x = _normal(rng, 20, 512)
    want = _linear(x, buf, 64, 128)
    x[3, 7], x[17, 500] = np.nan, np.inf
    got = _linear(x, buf, 64, 128)
    ok = np.ones(20, bool)
    ok[[3, 17]] = False
    assert np.array_equal(got[ok], want[ok])
    assert np.isnan(got[3]).all() and not np.isfinite(got[17]).any()


@pytest.mark.parametrize("h,a,g,tau,lens", [(512, 4, 2, [0, 0, 2], [0, 100, 63, 64]), (1024, 8, 8, [0, 1], [(29 * i) % 130 for i in range(70)])])
@pytest.mark.parametrize("form", ["slots", "paged", "noalloc"])
def test_decode_step_on_4_bit_weights(h, a, g, tau, lens, form):
    """The first layer on 4-bit weights, the others on bf16 ones: the decode step against the oracle on the weights that the
    codes stand for; taken off again, the step gives the bits it gave before."""
    w = small_workload(f"w4-h{h}-g{g}", len(tau), h, a, g, tau, seed=51)
    B, cap = len(lens), 192
    if form == "noalloc" and B > 64:
        pytest.skip("one call's scratch")
    say(f"[w4 decode] {w.name} B={B} {form}")
    dm = build_device_model(w, B, 1, cap, fill_cache_npos=max(lens))
    x = torch.empty((B, w.h), dtype=torch.bfloat16, device="cuda")
    kd.fill_decode_x(w, x.data_ptr(), B)
    lens_t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws, n = workspace(dm, kb.KVP_PHASE_DECODE, B)
    tab = torch.arange(B * 3, dtype=torch.int32, device="cuda").view(B, 3)
    if form == "paged":
        for l, (K, V) in dm.slots.items():      # the slots' contents in pages
            kp = K.view(B, g, 3, 64, 128).permute(1, 0, 2, 3, 4).reshape(g, B * 3, 64, 128).contiguous()
            vp = V.view(B, g, 128, 3, 64).permute(1, 0, 3, 2, 4).reshape(g, B * 3, 128, 64).contiguous()
            dm.tensors[f"kp{l}"], dm.tensors[f"vp{l}"] = kp, vp
            dm.model.kvp_set_kv_pool(l, kp.data_ptr(), vp.data_ptr(), B * 3)

    def step():
        y = torch.empty_like(x)
        if form == "paged":
            dm.model.kvp_decode_step_paged(x.data_ptr(), lens_t.data_ptr(), max(lens), tab.data_ptr(), 3, y.data_ptr(), B,
                                           ws.data_ptr(), n, _stream())
        elif form == "noalloc":
            dm.model.kvp_decode_step_noalloc(x.data_ptr(), lens_t.data_ptr(), max(lens), y.data_ptr(), B, _stream())
        else:
            dm.model.kvp_decode_step(x.data_ptr(), lens_t.data_ptr(), max(lens), y.data_ptr(), B, ws.data_ptr(), n, _stream())
        torch.cuda.synchronize()
        return y

    before = step()
    ows = oracle_weights(w)
    packed, exact = {}, {}
    for k in ("wq", "wk", "wv", "wo"):
        t = dm.tensors[k + "0"]
        codes, s = lr.w4_codes(t.float().cpu().numpy(), 128)
        packed[k], exact[k] = torch.from_numpy(lr.w4_pack(codes, s)).cuda(), lr.w4_weights(codes, s, 128)
    ows[0] = oat.LayerWeights(exact["wq"], exact["wk"], exact["wv"], exact["wo"])
    dm.model.kvp_set_layer_w4(0, *(packed[k].data_ptr() for k in ("wq", "wk", "wv", "wo")), 128)
    got = step()
    for b in (0, 1, B - 1):
        caches = {p: (ki.cache_contents(w, ki.KIND_KCACHE, p, b, lens[b]), ki.cache_contents(w, ki.KIND_VCACHE, p, b, lens[b]))
                  for p in dm.slots}
        yr = oat.decode_step(ki.decode_x(w, [b])[0], lens[b], ows, w.tau, caches, w.a, w.g, w.d_h, w.rope_base)[0]
        e = rel_err(to_np(got[b]), yr)
        say(f"  sequence {b}: {e:.3e}")
        assert e <= 2e-2, b
    dm.model.kvp_set_layer_w4(0, 0, 0, 0, 0, 0)
    assert torch.equal(step(), before)
