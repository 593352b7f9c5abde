"""Host-side checks of include/cdsgd_block.h that need no GPU: the library exports what the header declares, and bad arguments become status
codes before any HIP call."""
import ctypes
import os
import re

import pytest
import torch

from paper_2106_10796_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "cdsgd_block.h")
A = 0x7F0000000000          # addresses that are never dereferenced
F32, BF16, F16 = 0, 1, 2


def at(i):
    return A + i * 0x100000000


@pytest.fixture(scope="module")
def L():
    from paper_2106_10796_amd import build
    build.ensure_built()
    return B.lib()


def test_library_exports_every_declared_symbol(L):
    with open(HEADER) as fh:
        text = re.sub(r"/\*.*?\*/", "", fh.read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(cdsgd_[a-z0-9_]+)\s*\(", text)))
    assert len(names) == 12
    for name in names:
        assert getattr(L, name).argtypes is not None, "%s has no signature in the binding" % name


def test_sizes(L):
    for rows, cols, codes, scales in ((1, 1, 32, 1), (3, 32, 96, 3), (3, 33, 192, 6), (1 << 20, 4096, 1 << 32, 1 << 27)):
        assert L.cdsgd_mxint8_code_bytes(rows, cols) == codes and L.cdsgd_mxint8_scale_bytes(rows, cols) == scales
    assert L.cdsgd_block_norm_workspace(1, 4) == 32 and L.cdsgd_block_norm_workspace(0, 4) == 0 and L.cdsgd_block_norm_workspace(4, 16385) == 0


@pytest.mark.parametrize("want,over", [
    (B.ERR_NULL, dict(x=None)), (B.ERR_NULL, dict(codes=None)), (B.ERR_NULL, dict(scales=None)), (B.ERR_PARAM, dict(dtype=3)),
    (B.ERR_PARAM, dict(dtype=-1)), (B.ERR_SIZE, dict(rows=0)), (B.ERR_SIZE, dict(cols=0)), (B.ERR_SIZE, dict(rows=1 << 31)),
    (B.ERR_SIZE, dict(cols=1 << 31)), (B.ERR_SIZE, dict(ld=99)), (B.ERR_SIZE, dict(ld=(1 << 40) + 1)), (B.ERR_ALIGN, dict(x=at(0) + 1)),
    (B.ERR_ALIGN, dict(codes=at(1) + 8)), (B.ERR_ALIAS, dict(codes=at(0))), (B.ERR_ALIAS, dict(scales=at(1) + 127)),
    (B.ERR_ALIAS, dict(scales=at(0) + 99))])
def test_mxint8_refuses(L, want, over):
    a = dict(x=at(0), dtype=BF16, rows=10, cols=100, ld=100, codes=at(1), scales=at(2))
    a.update(over)
    assert L.cdsgd_mxint8_quantize(a["x"], a["dtype"], a["rows"], a["cols"], a["ld"], a["codes"], a["scales"], None) == want
    if over.get("scales") != at(1) + 127:       # (what dequantisation reads may overlap)
        assert L.cdsgd_mxint8_dequantize(a["codes"], a["scales"], a["rows"], a["cols"], a["x"], a["dtype"], a["ld"], None) == want


def _held(p=None, ld=0, codes=None, scales=None):
    return ctypes.byref(B.cdsgd_held(p, ld, codes, scales))


@pytest.mark.parametrize("want,over", [
    (B.ERR_NULL, dict(a=None)), (B.ERR_NULL, dict(u=None)), (B.ERR_NULL, dict(y=None)), (B.ERR_NULL, dict(a8=None)), (B.ERR_NULL, dict(us=None)),
    (B.ERR_PARAM, dict(act=2)), (B.ERR_PARAM, dict(dtype=5)), (B.ERR_SIZE, dict(rows=0)), (B.ERR_SIZE, dict(ld_u=99)), (B.ERR_ALIGN, dict(u=at(1) + 1)),
    (B.ERR_ALIGN, dict(a8=at(3) + 4)), (B.ERR_ALIAS, dict(y=at(0))), (B.ERR_ALIAS, dict(y=at(1) + 1998)), (B.ERR_ALIAS, dict(a8=at(1))),
    (B.ERR_ALIAS, dict(us=at(3) + 1279)), (B.ERR_ALIAS, dict(a8=at(4)))])
def test_gated_forward_refuses(L, want, over):
    v = dict(act=0, dtype=BF16, rows=10, a=at(0), u=at(1), y=at(2), ld_u=100, a8=at(3), as_=at(5), u8=at(4), us=at(6))
    v.update(over)
    assert L.cdsgd_gated_forward(v["act"], v["dtype"], v["rows"], 100, v["a"], 100, v["u"], v["ld_u"], v["y"], 100, v["a8"], v["as_"], v["u8"], v["us"],
                                 None) == want


@pytest.mark.parametrize("want,over", [
    (B.ERR_NULL, dict(dy=None)), (B.ERR_NULL, dict(a=None)), (B.ERR_NULL, dict(a=_held())), (B.ERR_NULL, dict(a=_held(codes=at(8)))),
    (B.ERR_PARAM, dict(a=_held(at(1), 100, at(8), at(9)))), (B.ERR_PARAM, dict(a=_held(codes=at(8), scales=at(9)))), (B.ERR_SIZE, dict(a=_held(at(1), 99))),
    (B.ERR_ALIGN, dict(a=_held(at(1) + 1, 100))), (B.ERR_ALIGN, dict(a=_held(codes=at(8) + 4, scales=at(9)))), (B.ERR_PARAM, dict(act=-1)),
    (B.ERR_NULL, dict(du=None)), (B.ERR_ALIAS, dict(da=at(1))), (B.ERR_ALIAS, dict(da=at(4))), (B.ERR_ALIAS, dict(du=at(0))), (B.ERR_ALIAS, dict(da=at(2) + 2)),
    # halves of one matrix overlap no more than its columns do
    (B.ERR_ALIAS, dict(da=at(4) + 198, ld_da=200, ld_du=200)), (B.ERR_ALIAS, dict(da=at(4) + 200, ld_da=201, ld_du=200))])
def test_gated_backward_refuses(L, want, over):
    v = dict(act=0, dy=at(0), a=_held(at(1), 100), u=_held(at(2), 100), da=at(3), du=at(4), ld_da=100, ld_du=100)
    v.update(over)
    assert L.cdsgd_gated_backward(v["act"], BF16, 10, 100, v["dy"], 100, v["a"], v["u"], v["da"], v["ld_da"], v["du"], v["ld_du"], None) == want


def _norm(**over):
    v = dict(dtype=BF16, stream_dtype=F32, rows=10, cols=100, weight=at(20), block_weight=at(21), gate=at(22), scale=0.5, eps=1e-6)
    v.update(over)
    return B.cdsgd_block_norm(**v)


BAD_NORMS = [(B.ERR_NULL, dict(weight=None)), (B.ERR_PARAM, dict(dtype=9)), (B.ERR_PARAM, dict(stream_dtype=F16)), (B.ERR_PARAM, dict(dtype=F32, stream_dtype=BF16)),
             (B.ERR_PARAM, dict(scale=float("inf"))), (B.ERR_PARAM, dict(eps=float("nan"))), (B.ERR_PARAM, dict(eps=-1e-9)), (B.ERR_SIZE, dict(rows=0)),
             (B.ERR_SIZE, dict(cols=0)), (B.ERR_SIZE, dict(cols=16385)), (B.ERR_SIZE, dict(rows=1 << 31)), (B.ERR_ALIGN, dict(gate=at(22) + 2))]


@pytest.mark.parametrize("want,norm,over", [(w, n, {}) for w, n in BAD_NORMS] + [(w, {}, o) for w, o in [
    (B.ERR_NULL, dict(h=None)), (B.ERR_NULL, dict(y=None)), (B.ERR_NULL, dict(rstd=None)), (B.ERR_NULL, dict(h_out=None)), (B.ERR_NULL, dict(h8=None)),
    (B.ERR_NULL, dict(bs=None)), (B.ERR_PARAM, dict(b=None)), (B.ERR_SIZE, dict(ld=99)), (B.ERR_ALIGN, dict(h=at(0) + 2)), (B.ERR_ALIGN, dict(y=at(3) + 1)),
    (B.ERR_ALIGN, dict(b8=at(7) + 8)), (B.ERR_ALIAS, dict(h_out=at(0))), (B.ERR_ALIAS, dict(y=at(1))), (B.ERR_ALIAS, dict(rstd=at(2))),
    (B.ERR_ALIAS, dict(h8=at(7))), (B.ERR_ALIAS, dict(rstd=at(20)))]])
def test_block_norm_forward_refuses(L, want, norm, over):
    v = dict(h=at(0), b=at(1), h_out=at(2), y=at(3), rstd=at(4), h8=at(5), hs=at(6), b8=at(7), bs=at(8), ld=100)
    v.update(over)
    assert L.cdsgd_block_norm_forward(ctypes.byref(_norm(**norm)), v["h"], 100, v["b"], v["ld"], v["h_out"], 100, v["y"], 100, v["rstd"], v["h8"], v["hs"],
                                      v["b8"], v["bs"], None) == want


def test_a_norm_without_a_block_takes_nothing_of_one(L):
    none = dict(block_weight=None, gate=None)
    for norm, h_out, b8 in ((_norm(**none), at(2), None), (_norm(**none), None, at(7)), (_norm(gate=None), None, None), (_norm(block_weight=None), None, None)):
        assert L.cdsgd_block_norm_forward(ctypes.byref(norm), at(0), 100, None, 0, h_out, 100, at(3), 100, at(4), None, None, b8, b8 and at(8),
                                          None) == B.ERR_PARAM
    assert L.cdsgd_block_norm_forward(None, at(0), 100, None, 0, None, 0, at(3), 100, at(4), None, None, None, None, None) == B.ERR_NULL


@pytest.mark.parametrize("want,norm,over", [(w, n, {}) for w, n in BAD_NORMS] + [(w, {}, o) for w, o in [
    (B.ERR_NULL, dict(dy=None)), (B.ERR_NULL, dict(h=None)), (B.ERR_NULL, dict(h=_held())), (B.ERR_NULL, dict(rstd=None)), (B.ERR_NULL, dict(dh=None)),
    (B.ERR_NULL, dict(db=None)), (B.ERR_NULL, dict(dw=None)), (B.ERR_NULL, dict(dw_b=None)), (B.ERR_NULL, dict(dgate=None)), (B.ERR_NULL, dict(room=None)),
    (B.ERR_PARAM, dict(b=_held())), (B.ERR_SIZE, dict(room_bytes=8000 - 1)), (B.ERR_SIZE, dict(h=_held(at(2), 99))), (B.ERR_ALIGN, dict(room=at(14) + 8)),
    (B.ERR_ALIAS, dict(dh=at(1))), (B.ERR_ALIAS, dict(db=at(0))), (B.ERR_ALIAS, dict(dw=at(11))), (B.ERR_ALIAS, dict(room=at(2))),
    (B.ERR_ALIAS, dict(dgate=at(22))), (B.ERR_ALIAS, dict(dh=at(3)))]])
def test_block_norm_backward_refuses(L, want, norm, over):
    v = dict(dy=at(0), dt=at(1), h=_held(at(2), 100), b=_held(at(3), 100), rstd=at(4), dh=at(8), db=at(9), dw=at(10), dw_b=at(11), dgate=at(12), room=at(14),
             room_bytes=8000)
    v.update(over)
    assert L.cdsgd_block_norm_backward(ctypes.byref(_norm(**norm)), v["dy"], 100, v["dt"], 100, v["h"], v["b"], v["rstd"], v["dh"], 100, v["db"], 100, v["dw"],
                                       v["dw_b"], v["dgate"], v["room"], v["room_bytes"], None) == want


def test_gradients_of_weights_that_are_not_there(L):
    for norm, dw_b, dgate in ((_norm(block_weight=None), at(11), at(12)), (_norm(gate=None), at(11), at(12))):
        assert L.cdsgd_block_norm_backward(ctypes.byref(norm), at(0), 100, None, 0, _held(at(2), 100), _held(at(3), 100), at(4), at(8), 100, at(9), 100, at(10),
                                           dw_b, dgate, at(14), 8000, None) == B.ERR_PARAM


def _batch(**over):
    v = dict(dtype=BF16, causal=1, tokens_q=100, tokens_k=100, num_seqs=3, starts_q=at(30), starts_k=None, heads=8, kv_heads=2, dim=64, scale=0.125)
    v.update(over)
    return B.cdsgd_attention(**v)


BAD_BATCHES = [(B.ERR_PARAM, dict(dtype=F32)), (B.ERR_PARAM, dict(causal=2)), (B.ERR_PARAM, dict(kv_heads=3)), (B.ERR_PARAM, dict(starts_q=None)),
               (B.ERR_PARAM, dict(starts_q=None, starts_k=at(31), num_seqs=1)), (B.ERR_PARAM, dict(scale=0.0)), (B.ERR_PARAM, dict(scale=-1.0)),
               (B.ERR_PARAM, dict(scale=float("nan"))), (B.ERR_PARAM, dict(scale=1e300)), (B.ERR_SIZE, dict(tokens_q=0)), (B.ERR_SIZE, dict(tokens_k=0)),
               (B.ERR_SIZE, dict(tokens_k=1 << 31)), (B.ERR_SIZE, dict(num_seqs=0)), (B.ERR_SIZE, dict(num_seqs=1 << 24)), (B.ERR_SIZE, dict(heads=0)),
               (B.ERR_SIZE, dict(kv_heads=0)), (B.ERR_SIZE, dict(heads=65536)), (B.ERR_SIZE, dict(dim=0)), (B.ERR_SIZE, dict(dim=12)), (B.ERR_SIZE, dict(dim=136)),
               (B.ERR_SIZE, dict(tokens_q=(1 << 31) - 1)), (B.ERR_ALIGN, dict(starts_q=at(30) + 2)), (B.ERR_ALIGN, dict(starts_k=at(31) + 1))]


@pytest.mark.parametrize("want,batch,over", [(w, b, {}) for w, b in BAD_BATCHES] + [(w, {}, o) for w, o in [
    (B.ERR_NULL, dict(q=None)), (B.ERR_NULL, dict(k=None)), (B.ERR_NULL, dict(v=None)), (B.ERR_NULL, dict(out=None)), (B.ERR_SIZE, dict(ld_q=504)),
    (B.ERR_SIZE, dict(ld_q=(1 << 20) + 8)), (B.ERR_ALIGN, dict(ld_q=516)), (B.ERR_ALIGN, dict(k=at(1) + 8)), (B.ERR_ALIGN, dict(lse=at(4) + 1)),
    (B.ERR_ALIAS, dict(out=at(0))), (B.ERR_ALIAS, dict(out=at(2) + 1024)), (B.ERR_ALIAS, dict(lse=at(1))), (B.ERR_ALIAS, dict(lse=at(30) + 12)),
    (B.ERR_ALIAS, dict(lse=at(3) + 512))]])
def test_attention_forward_refuses(L, want, batch, over):
    v = dict(q=at(0), k=at(1), v=at(2), out=at(3), lse=at(4), ld_q=512)
    v.update(over)
    assert L.cdsgd_attention_forward(ctypes.byref(_batch(**batch)), v["q"], v["ld_q"], v["k"], 128, v["v"], 128, v["out"], 512, v["lse"], None, 0, None) == want


@pytest.mark.parametrize("want,batch,over", [(w, b, {}) for w, b in BAD_BATCHES] + [(w, {}, o) for w, o in [
    (B.ERR_NULL, dict(dout=None)), (B.ERR_NULL, dict(out=None)), (B.ERR_NULL, dict(lse=None)), (B.ERR_NULL, dict(dq=None)), (B.ERR_NULL, dict(dk=None)),
    (B.ERR_NULL, dict(dv=None)), (B.ERR_NULL, dict(room=None)), (B.ERR_SIZE, dict(room_bytes=100 * 8 * 12 - 1)), (B.ERR_ALIGN, dict(room=at(9) + 8)),
    (B.ERR_ALIAS, dict(dq=at(5))), (B.ERR_ALIAS, dict(dk=at(7))), (B.ERR_ALIAS, dict(dk=at(8) + 128)), (B.ERR_ALIAS, dict(dv=at(0))), (B.ERR_ALIAS, dict(dk=at(4))),
    (B.ERR_ALIAS, dict(room=at(3))), (B.ERR_ALIAS, dict(dk=at(30)))]])
def test_attention_backward_refuses(L, want, batch, over):
    v = dict(q=at(0), k=at(1), v=at(2), out=at(3), lse=at(4), dout=at(5), dq=at(6), dk=at(7), dv=at(8), room=at(9), room_bytes=100 * 8 * 12)
    v.update(over)
    if over == dict(dk=at(7)):
        v["dq"] = at(7)
    assert L.cdsgd_attention_backward(ctypes.byref(_batch(**batch)), v["dout"], 512, v["q"], 512, v["k"], 128, v["v"], 128, v["out"], 512, v["lse"], v["dq"], 512,
                                      v["dk"], 128, v["dv"], 128, v["room"], v["room_bytes"], None) == want


def test_split_keys_need_their_workspace(L):
    """A few tokens over many keys; batches that need none say 0, as do bad ones."""
    few = _batch(tokens_q=1, tokens_k=100000, num_seqs=1)
    need = L.cdsgd_attention_workspace(ctypes.byref(few), 0)
    assert need > 0 and need % 16 == 0
    args = [at(0), 512, at(1), 128, at(2), 128, at(3), 512, at(4)]
    assert L.cdsgd_attention_forward(ctypes.byref(few), *args, None, 0, None) == B.ERR_NULL
    assert L.cdsgd_attention_forward(ctypes.byref(few), *args, at(9), need - 1, None) == B.ERR_SIZE
    assert L.cdsgd_attention_forward(ctypes.byref(few), *args, at(9) + 4, need, None) == B.ERR_ALIGN
    assert L.cdsgd_attention_forward(ctypes.byref(few), *args, at(3), need, None) == B.ERR_ALIAS
    assert L.cdsgd_attention_workspace(ctypes.byref(_batch()), 0) == 0
    assert L.cdsgd_attention_workspace(ctypes.byref(_batch(dim=12)), 1) == 0 and L.cdsgd_attention_workspace(None, 1) == 0


def test_binding_says_what_is_wrong():
    x, w = torch.zeros(4, 32, dtype=torch.bfloat16), torch.zeros(32)
    with pytest.raises(TypeError, match="x must be a CUDA matrix"):
        B.cdsgd_mxint8_quantize(x, B.new_mxint8(4, 32, device="cpu"))
    with pytest.raises(TypeError, match="q must be an Mxint8"):
        B.cdsgd_mxint8_dequantize(x, x)
    with pytest.raises(TypeError, match="a must be a CUDA matrix"):
        B.cdsgd_gated_forward(x, x, x)
    with pytest.raises(TypeError, match="weight must be a contiguous CUDA tensor"):
        B.BlockNorm(w)
    with pytest.raises(TypeError, match="q must be a CUDA tensor"):
        B.cdsgd_attention_forward(x, x, x, x)
    with pytest.raises(ValueError, match="act must be one of"):
        B._act("relu")


@pytest.mark.gpu
def test_binding_says_what_is_wrong_on_the_gpu():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    x = bf(4, 64)
    with pytest.raises(ValueError, match="u is a matrix of 4 by 63"):
        B.cdsgd_gated_forward(x, bf(4, 63), bf(4, 64))
    with pytest.raises(TypeError, match="y must have the type of the others"):
        B.cdsgd_gated_forward(x, bf(4, 64), torch.zeros(4, 64, device="cuda"))
    with pytest.raises(TypeError, match="rows of u must be contiguous"):
        B.cdsgd_gated_forward(x, bf(4, 128)[:, ::2], bf(4, 64))
    with pytest.raises(ValueError, match="a8 is a matrix of 3 by 64"):
        B.cdsgd_gated_forward(x, bf(4, 64), bf(4, 64), B.new_mxint8(3, 64), B.new_mxint8(4, 64))
    with pytest.raises(B.CdsgdError) as e:
        B.cdsgd_gated_forward(x, bf(4, 64), bf(4, 64), B.new_mxint8(4, 64))
    assert e.value.status == B.ERR_NULL
    norm = B.BlockNorm(torch.ones(64, device="cuda"))
    with pytest.raises(ValueError, match="y has 60 columns, expected 64"):
        norm.forward(x, bf(4, 60), torch.zeros(2, 4, device="cuda"))
    with pytest.raises(ValueError, match="rstd has 4 elements, expected 8"):
        norm.forward(x, bf(4, 64), torch.zeros(4, device="cuda"))
    q, k = bf(9, 4, 64), bf(9, 2, 64)
    out, lse = bf(9, 4, 64), torch.zeros(4, 9, device="cuda")
    for bad, error, match in ((dict(v=bf(9, 2, 72)), ValueError, "v has shape"), (dict(out=bf(9, 2, 64)), ValueError, "out has shape"),
                              (dict(k=k.half()), TypeError, "k must have the type"), (dict(q=bf(9, 64, 4).transpose(1, 2)), TypeError, "must lie in a row"),
                              (dict(lse=lse[:3]), ValueError, "lse has 27 elements"),
                              (dict(starts=torch.tensor([0, 9], device="cuda")), TypeError, "starts must be a contiguous CUDA vector of int32"),
                              (dict(starts_k=torch.tensor([0, 9], dtype=torch.int32, device="cuda")), ValueError, "starts_k without starts"),
                              (dict(q=bf(9, 4, 32), out=bf(9, 4, 32)), ValueError, "heads of 32 and of 64")):
        with pytest.raises(error, match=match):
            B.cdsgd_attention_forward(**{**dict(q=q, k=k, v=k.clone(), out=out, lse=lse), **bad})
    with pytest.raises(B.CdsgdError) as e:
        B.cdsgd_attention_forward(q, bf(9, 3, 64), bf(9, 3, 64), out, lse)
    assert e.value.status == B.ERR_PARAM
    with pytest.raises(B.CdsgdError) as e:
        B.cdsgd_attention_backward(out, q, k, k.clone(), out.clone(), lse, q.clone(), k.clone(), k.clone())
    assert e.value.status == B.ERR_NULL
