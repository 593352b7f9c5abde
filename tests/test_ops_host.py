"""Host-side checks of include/cdsgd_ops.h that need no GPU: the library exports what the header declares, and bad arguments
become status codes before any HIP call."""
import ctypes
import os
import re

import pytest

from paper_2106_10796_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "cdsgd_ops.h")
A = 0x7F0000000000          # addresses that are never dereferenced
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def L():
    from paper_2106_10796_amd import build
    build.ensure_built()
    return B.lib()


def _header():
    with open(HEADER) as fh:
        return re.sub(r"/\*.*?\*/", "", fh.read(), flags=re.S)


def test_library_exports_every_declared_symbol(L):
    names = sorted(set(re.findall(r"\b(cdsgd_[a-z0-9_]+)\s*\(", _header())))
    assert len(names) >= 10
    for name in names:
        fn = getattr(L, name)
        assert fn.argtypes is not None, "%s has no signature in the binding" % name


def test_constants(L):
    assert int(re.search(r"#define CDSGD_STATE_BLOCK (\d+)", _header())[1]) == B.STATE_BLOCK
    for n, blocks in ((1, 1), (256, 1), (257, 2), (1 << 33, 1 << 25)):
        assert L.cdsgd_state_blocks(n) == blocks


def _adamw(n=1000, bits=32, i=0, **over):
    at = A + i * 0x1000000
    t = dict(weight=at, weight16=None, grad=at + 0x100000, m=at + 0x200000, v=at + 0x300000,
             m_scale=at + 0x400000 if bits == 8 else None, v_scale=at + 0x500000 if bits == 8 else None, n=n, weight_decay=0.1)
    t.update(over)
    return B.cdsgd_adamw_tensor(**t)


def _create(L, tensors, dtype=F32, bits=32):
    out = ctypes.c_void_p(1)
    arr = (B.cdsgd_adamw_tensor * max(len(tensors), 1))(*tensors)
    st = L.cdsgd_adamw_plan_create(arr, len(tensors), dtype, bits, ctypes.byref(out))
    assert out.value is None
    return st


@pytest.mark.parametrize("want,dtype,bits,over", [
    (B.ERR_NULL, F32, 32, dict(weight=None)), (B.ERR_NULL, F32, 32, dict(grad=None)),
    (B.ERR_NULL, F32, 32, dict(m=None)), (B.ERR_NULL, F32, 32, dict(v=None)),
    (B.ERR_NULL, F32, 8, dict(m_scale=None)), (B.ERR_NULL, F32, 8, dict(v_scale=None)),
    (B.ERR_PARAM, F32, 32, dict(m_scale=A + 0x700000)), (B.ERR_SIZE, F32, 32, dict(n=0)), (B.ERR_SIZE, F32, 32, dict(n=1 << 50)),
    (B.ERR_SIZE, F32, 32, dict(n=1 << 39)),
    (B.ERR_PARAM, F32, 32, dict(weight_decay=-0.1)), (B.ERR_PARAM, F32, 32, dict(weight_decay=float("nan"))),
    (B.ERR_PARAM, F32, 32, dict(weight16=A + 0x700000)),           # a copy no narrower than the weights
    (B.ERR_PARAM, 3, 32, {}), (B.ERR_PARAM, F32, 16, {}),
    (B.ERR_ALIGN, F32, 32, dict(weight=A + 4)), (B.ERR_ALIGN, BF16, 32, dict(grad=A + 0x100008)),
    (B.ERR_ALIGN, F32, 8, dict(m=A + 0x200001)), (B.ERR_ALIGN, BF16, 8, dict(weight16=A + 0x700002)),
    (B.ERR_ALIAS, F32, 32, dict(m=A)), (B.ERR_ALIAS, F32, 32, dict(grad=A + 16)), (B.ERR_ALIAS, F32, 8, dict(m_scale=A + 0x200000)),
    (B.ERR_ALIAS, F32, 8, dict(m_scale=A + 0x200000 + 999)), (B.ERR_ALIAS, F32, 8, dict(v_scale=A + 0x400003)),
    (B.ERR_ALIAS, F16, 32, dict(weight16=A + 0x100000 + 1984)),
])
def test_adamw_plan_refuses(L, want, dtype, bits, over):
    assert _create(L, [_adamw(bits=bits, **over)], dtype, bits) == want
    other = {k: (v + 0x1000000 if isinstance(v, int) and v >= A else v) for k, v in over.items()}
    if "weight16" not in over:
        assert _create(L, [_adamw(bits=bits), _adamw(bits=bits, i=1, **other)], dtype, bits) == want


@pytest.mark.parametrize("over", [dict(weight=A), dict(m=A + 0x300000), dict(v=A + 0x300000 + 3984), dict(grad=A), dict(m=A + 0x100000)])
def test_adamw_plan_refuses_what_two_tensors_share(L, over):
    assert _create(L, [_adamw(), _adamw(i=1, **over)]) == B.ERR_ALIAS
    assert _create(L, [_adamw(i=1, **over), _adamw(i=2), _adamw()]) == B.ERR_ALIAS


def test_adamw_refuses_more(L):
    assert _create(L, []) == B.ERR_SIZE
    assert L.cdsgd_adamw_plan_create(None, 1, F32, 32, ctypes.byref(ctypes.c_void_p())) == B.ERR_NULL
    assert L.cdsgd_adamw_plan_create((B.cdsgd_adamw_tensor * 1)(_adamw()), 1, F32, 32, None) == B.ERR_NULL
    # a 16-bit copy of some tensors alone
    assert _create(L, [_adamw(), _adamw(i=1, weight16=A + 0x1700000)], BF16) == B.ERR_PARAM
    assert L.cdsgd_adamw_step(None, 1, 1e-3, 0.9, 0.999, 1e-8, 1.0, 0, None, None) == B.ERR_NULL
    assert L.cdsgd_adamw_grad_norm(None, 1.0, 1.0, A, None) == B.ERR_NULL
    assert L.cdsgd_adamw_bind_readout(None, None, None, 0) == B.ERR_NULL
    assert L.cdsgd_adamw_read_states(None, None) == B.ERR_NULL
    assert L.cdsgd_adamw_plan_destroy(None) == B.OK


def test_grad_norm_refuses(L):
    out = ctypes.c_void_p(1)
    one, n = (ctypes.c_void_p * 1)(A), (ctypes.c_size_t * 1)(100)
    create = L.cdsgd_grad_norm_create
    assert create(None, n, 1, F32, ctypes.byref(out)) == B.ERR_NULL
    assert create(one, None, 1, F32, ctypes.byref(out)) == B.ERR_NULL
    assert create(one, n, 1, F32, None) == B.ERR_NULL
    assert create(one, n, 0, F32, ctypes.byref(out)) == B.ERR_SIZE
    assert create(one, n, 1, 7, ctypes.byref(out)) == B.ERR_PARAM
    assert create((ctypes.c_void_p * 1)(None), n, 1, F32, ctypes.byref(out)) == B.ERR_NULL
    assert create((ctypes.c_void_p * 1)(A + 8), n, 1, F32, ctypes.byref(out)) == B.ERR_ALIGN
    for bad in (0, 1 << 50, 1 << 39):
        assert create(one, (ctypes.c_size_t * 1)(bad), 1, F32, ctypes.byref(out)) == B.ERR_SIZE
    assert out.value is None
    assert L.cdsgd_grad_norm_compute(None, 1.0, 1.0, A, None) == B.ERR_NULL
    assert L.cdsgd_grad_norm_destroy(None) == B.OK


def test_binding_says_what_is_wrong(L):
    import torch
    t = dict(weight=torch.zeros(4), grad=torch.zeros(4), m=torch.zeros(4), v=torch.zeros(4))
    with pytest.raises(TypeError, match="weight must be"):
        B.AdamWPlan([t])
    with pytest.raises(TypeError, match="gradients must be"):
        B.AdamWPlan([t], grad_dtype=torch.float64)
    with pytest.raises(TypeError, match="gradients must be"):
        B.GradNorm([torch.zeros(4, dtype=torch.float64)])
    with pytest.raises(TypeError, match=r"grads\[0\] must be"):
        B.GradNorm([torch.zeros(4)])
    with pytest.raises(B.CdsgdError):
        B.GradNorm([])


def test_mxfp4_sizes(L):
    for r, c, g in ((1, 1, 1), (3, 128, 1), (3, 129, 2), (100000, 25088, 196)):
        assert L.cdsgd_mxfp4_code_bytes(r, c) == r * g * 64 and L.cdsgd_mxfp4_scale_bytes(r, c) == r * g * 4


Q = [A + i * 0x10000000 for i in range(8)]     # buffers far apart


def test_mxfp4_quantize_refuses(L):
    f = L.cdsgd_mxfp4_quantize
    ok = [Q[0], F32, 100, 200, 200, Q[1], Q[2], Q[3], Q[4], None]

    def st(**over):
        names = ("x", "dtype", "rows", "cols", "ld", "codes", "scales", "codes_t", "scales_t", "stream")
        return f(*[over.get(n, v) for n, v in zip(names, ok)])
    for over in (dict(x=None), dict(codes=None), dict(scales=None), dict(codes_t=None), dict(scales_t=None),
                 dict(codes=None, scales=None, codes_t=None, scales_t=None)):
        assert st(**over) == B.ERR_NULL, over
    assert st(dtype=3) == B.ERR_PARAM
    for over in (dict(rows=0), dict(cols=0), dict(rows=1 << 31), dict(cols=1 << 31), dict(ld=199), dict(ld=1 << 50)):
        assert st(**over) == B.ERR_SIZE, over
    for over in (dict(x=Q[0] + 2), dict(dtype=BF16, x=Q[0] + 1), dict(codes=Q[1] + 8), dict(scales=Q[2] + 2), dict(codes_t=Q[3] + 4),
                 dict(scales_t=Q[4] + 1)):
        assert st(**over) == B.ERR_ALIGN, over
    for over in (dict(codes=Q[0]), dict(codes_t=Q[1]), dict(scales=Q[1] + 100 * 128 - 4), dict(scales_t=Q[3]),
                 dict(codes=Q[0] + 4 * (99 * 200 + 200) // 16 * 16 - 16)):
        assert st(**over) == B.ERR_ALIAS, over


def test_mxfp4_dequantize_refuses(L):
    f = L.cdsgd_mxfp4_dequantize
    assert f(None, Q[1], 10, 20, Q[2], F32, 20, None) == B.ERR_NULL
    assert f(Q[0], None, 10, 20, Q[2], F32, 20, None) == B.ERR_NULL
    assert f(Q[0], Q[1], 10, 20, None, F32, 20, None) == B.ERR_NULL
    assert f(Q[0], Q[1], 10, 20, Q[2], 5, 20, None) == B.ERR_PARAM
    assert f(Q[0], Q[1], 0, 20, Q[2], F32, 20, None) == B.ERR_SIZE
    assert f(Q[0], Q[1], 10, 20, Q[2], F32, 19, None) == B.ERR_SIZE
    assert f(Q[0] + 4, Q[1], 10, 20, Q[2], F32, 20, None) == B.ERR_ALIGN
    assert f(Q[0], Q[1] + 2, 10, 20, Q[2], F32, 20, None) == B.ERR_ALIGN
    assert f(Q[0], Q[1], 10, 20, Q[2] + 2, F32, 20, None) == B.ERR_ALIGN
    assert f(Q[0], Q[1], 10, 20, Q[0] + 16, F32, 20, None) == B.ERR_ALIAS
    assert f(Q[0], Q[1], 10, 20, Q[1] + 36, F32, 20, None) == B.ERR_ALIAS


def test_mxfp4_matmul_refuses(L):
    names = ("ac", "as_", "bc", "bs", "M", "N", "K", "out", "dtype", "ld", "add", "ws", "wb", "stream")
    ok = [Q[0], Q[1], Q[2], Q[3], 300, 400, 500, Q[4], F32, 400, 0, Q[5], 1 << 27, None]

    def st(**over):
        return L.cdsgd_mxfp4_matmul(*[over.get(n, v) for n, v in zip(names, ok)])
    for n in ("ac", "as_", "bc", "bs", "out"):
        assert st(**{n: None}) == B.ERR_NULL
    assert st(dtype=9) == B.ERR_PARAM
    for over in (dict(M=0), dict(N=0), dict(K=0), dict(M=(1 << 29) + 1), dict(N=(1 << 29) + 1, ld=1 << 30), dict(K=(1 << 24) + 1), dict(ld=399)):
        assert st(**over) == B.ERR_SIZE, over
    for over in (dict(ac=Q[0] + 8), dict(bc=Q[2] + 1), dict(as_=Q[1] + 2), dict(bs=Q[3] + 1), dict(out=Q[4] + 2), dict(ws=Q[5] + 8)):
        assert st(**over) == B.ERR_ALIGN, over
    for over in (dict(out=Q[0]), dict(out=Q[1] + 4), dict(out=Q[2] - 4), dict(out=Q[3])):
        assert st(**over) == B.ERR_ALIAS, over
    # a product that needs a workspace
    shapes = [(m, n, k) for m in (1, 16, 64, 300) for n in (128, 400, 4096) for k in (4096, 25088)] + [(600, 800, 16500)]
    shapes = [s for s in shapes if L.cdsgd_mxfp4_matmul_workspace(*s)]
    assert shapes
    for M, N, K in shapes:
        need = L.cdsgd_mxfp4_matmul_workspace(M, N, K)
        assert need % 16 == 0
        assert st(M=M, N=N, K=K, ld=N, ws=None, wb=0) == B.ERR_NULL
        assert st(M=M, N=N, K=K, ld=N, wb=need - 1) == B.ERR_SIZE
        assert st(M=M, N=N, K=K, ld=N, ws=Q[4], wb=need) == B.ERR_ALIAS
        assert st(M=M, N=N, K=K, ld=N, ws=Q[2], wb=need) == B.ERR_ALIAS


def test_mxfp4_binding_says_what_is_wrong(L):
    import torch
    q = B.new_mxfp4(3, 130, device="cpu")
    assert q.codes.shape == (3, 128) and q.scales.shape == (2, 3, 4)
    with pytest.raises(TypeError, match="x must be a CUDA matrix"):
        B.cdsgd_mxfp4_quantize(torch.zeros(3, 130), q)
    with pytest.raises(TypeError, match="q must be an Mxfp4"):
        B.cdsgd_mxfp4_dequantize(q.codes, torch.zeros(3, 130))
    with pytest.raises(TypeError, match=r"a.codes must be"):
        B.cdsgd_mxfp4_matmul(q, q, torch.zeros(3, 3))
    assert B.new_mxfp4_workspace([]) is None
    wide = B.Mxfp4(q.codes.long(), q.scales, 3, 130)
    assert wide.codes.dtype == torch.uint8 and torch.equal(wide.codes, q.codes) and wide.scales is q.scales


def test_native_calls_decline_what_is_not_plainly_good(L):
    import torch
    native = B._native()
    if isinstance(native, B._Declines):
        pytest.skip("the native calls are not there")

    def no_stream():
        raise AssertionError("asked for a stream though an argument is not good")

    f, q = torch.zeros(4, 256), B.new_mxfp4(4, 256, device="cpu")
    two = torch.zeros(2)
    for got in (native.mxfp4_quantize(f, q, None, no_stream), native.mxfp4_quantize(None, q, None, no_stream), native.mxfp4_quantize(f, q, None),
                native.mxfp4_dequantize(q, f, no_stream), native.mxfp4_dequantize(tuple(q), f, no_stream),
                native.mxfp4_matmul(q, q, f, None, False, no_stream), native.mxfp4_matmul(q, q, f, None, 0, no_stream),
                native.adamw_step(None, 1, 0.1, 0.9, 0.999, 1e-8, 1.0, 0, None, no_stream),
                native.adamw_step(0, 1, 0.1, 0.9, 0.999, 1e-8, 1.0, 0, None, no_stream),
                native.adamw_step(16, 1, 1, 0.9, 0.999, 1e-8, 1.0, 0, None, no_stream),
                native.adamw_step(16, 1, 0.1, 0.9, 0.999, 1e-8, 1.0, 0, two, no_stream),
                native.adamw_grad_norm(None, two, 1.0, 1.0, no_stream), native.adamw_grad_norm(16, two, 1.0, 1.0, no_stream),
                native.grad_norm_compute(None, two, 1.0, 1.0, no_stream), native.adamw_read_states(None, no_stream)):
        assert got == -1
