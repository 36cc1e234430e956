"""Thin binding of include/rv_kernels.h (per-kernel entry points; marshalling only)."""
import ctypes
import struct
from contextlib import nullcontext
from functools import lru_cache

import torch

from . import _lib
from .api import _check, _flat, _on, _ptr, _stream_handle

EPI_BF16, EPI_BF16_BIAS, EPI_F32_BIAS_RESID, EPI_BF16_BIAS_GELU, EPI_BF16_DGELU, EPI_F32, EPI_F32_BIAS_RESID_BF16 = range(7)


def gemm_bf16(A, a_kmajor, B, b_kmajor, M, N, K, epilogue, out, out2=None, bias=None, resid=None, zin=None,
              tile=0, stream=None):
    lda = A.stride(0); ldb = B.stride(0)
    _check(_lib.lib().rv_k_gemm_bf16(_ptr(A), lda, int(a_kmajor), _ptr(B), ldb, int(b_kmajor), M, N, K, epilogue,
                                     _ptr(out), out.stride(0), _ptr(out2), _ptr(bias), _ptr(resid),
                                     resid.stride(0) if resid is not None else 0, _ptr(zin), tile,
                                     _stream_handle(stream)))
    return out


def gemm_bf16_blocks(A, a_blocks, a_kmajor, B, b_blocks, b_kmajor, M, N, K, epilogue, out, out2=None, out_blocks=0, bias=None, resid=None,
                     zin=None, tile=0, parts=0, stream=None):
    """rv_k_gemm_bf16_blocks: operands and results in rows or in blocks of 32 columns."""
    _check(_lib.lib().rv_k_gemm_bf16_blocks(_ptr(A), int(a_blocks), int(a_kmajor), _ptr(B), int(b_blocks), int(b_kmajor), M, N, K, epilogue,
                                            _ptr(out), _ptr(out2), int(out_blocks), _ptr(bias), _ptr(resid), _ptr(zin), tile, parts,
                                            _stream_handle(stream)))
    return out


def stage_less_work(stage):
    """rv_k_stage_less_work: the stage's smaller work buffer."""
    _check(_lib.lib().rv_k_stage_less_work(stage._h))


def gemm_part(A, B, b_kmajor, M, N, K, tile, parts, stream=None):
    """rv_k_gemm_part: fp32 [parts, M, N], the product's sums over `parts` stretches of the contraction."""
    part = torch.full((parts, M, N), float("nan"), dtype=torch.float32, device="cuda")
    _check(_lib.lib().rv_k_gemm_part(_ptr(A), A.stride(0), _ptr(B), B.stride(0), int(b_kmajor), M, N, K, tile, parts, _ptr(part),
                                     _stream_handle(stream)))
    return part


def gemm_wgrad_grouped(xs, dys, outs, stream=None):
    """rv_k_gemm_wgrad_grouped: outs[i] (fp32 [M_i, N_i]) = xs[i]^T @ dys[i]; xs[i] is [K, M_i], dys[i] is [K, N_i]."""
    n = len(xs)
    K = xs[0].shape[0]
    vp = (ctypes.c_void_p * n); i64 = (ctypes.c_int64 * n); i32 = (ctypes.c_int * n)
    X = vp(*[_ptr(x) for x in xs]); Y = vp(*[_ptr(y) for y in dys]); O = vp(*[_ptr(o) for o in outs])
    lda = i64(*[x.stride(0) for x in xs]); ldb = i64(*[y.stride(0) for y in dys])
    M = i32(*[x.shape[1] for x in xs]); N = i32(*[y.shape[1] for y in dys])
    _check(_lib.lib().rv_k_gemm_wgrad_grouped(n, X, lda, Y, ldb, M, N, K, O, _stream_handle(stream)))
    return outs


def gemm_wgrad_update(xs, dys, outs=None, w=None, ver=None, eta=0.0, stream=None):
    """rv_k_gemm_wgrad_update: the products of gemm_wgrad_grouped in the form a decoder stage launches, with the
    update of the fp32 masters w[i] and bf16 versions ver[i] where given."""
    n = len(xs)
    vp = (ctypes.c_void_p * n); i64 = (ctypes.c_int64 * n); i32 = (ctypes.c_int * n)
    arr = lambda ts: vp(*[_ptr(t) for t in ts]) if ts is not None else None
    _check(_lib.lib().rv_k_gemm_wgrad_update(n, arr(xs), i64(*[x.stride(0) for x in xs]), arr(dys),
                                             i64(*[y.stride(0) for y in dys]), i32(*[x.shape[1] for x in xs]),
                                             i32(*[y.shape[1] for y in dys]), xs[0].shape[0], arr(outs), arr(w), arr(ver),
                                             eta, _stream_handle(stream)))
    return outs


def layernorm_fwd(x, gamma, beta, eps, xcopy=None, stream=None):
    T, d = x.shape
    y = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    mean = torch.empty(T, dtype=torch.float32, device="cuda"); rstd = torch.empty_like(mean)
    _check(_lib.lib().rv_k_layernorm_fwd(_ptr(x), 1 if x.dtype == torch.bfloat16 else 0, _ptr(xcopy), _ptr(gamma),
                                         _ptr(beta), _ptr(y), _ptr(mean), _ptr(rstd), T, d, eps,
                                         _stream_handle(stream)))
    return y, mean, rstd


def layernorm_fwd_parts(part, bias, resid, gamma, beta, eps, stream=None):
    """(xsum, y, mean, rstd); without gamma: (xsum, xsum rounded to bf16)."""
    S, T, d = part.shape
    xsum, y = torch.empty(T, d, dtype=torch.float32, device="cuda"), torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    ln = gamma is not None
    mean, rstd = (torch.empty(T, dtype=torch.float32, device="cuda") if ln else None for _ in range(2))
    _check(_lib.lib().rv_k_layernorm_fwd_parts(_ptr(part), S, _ptr(bias), _ptr(resid), _ptr(xsum), _ptr(gamma), _ptr(beta),
                                               _ptr(y if ln else None), _ptr(mean), _ptr(rstd), _ptr(None if ln else y), T, d, eps,
                                               _stream_handle(stream)))
    return (xsum, y, mean, rstd) if ln else (xsum, y)


def layernorm_bwd_parts(dy_part, x, mean, rstd, gamma, dres, rows, stream=None):
    """(dx, its bf16 rounding, column sums fp32 [ceil(T / rows), 3, d])."""
    S, T, d = dy_part.shape
    dx, dx16 = torch.empty(T, d, dtype=torch.float32, device="cuda"), torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    part = torch.empty((T + rows - 1) // rows, 3, d, dtype=torch.float32, device="cuda")
    _check(_lib.lib().rv_k_layernorm_bwd_parts(_ptr(dy_part), S, _ptr(x), _ptr(mean), _ptr(rstd), _ptr(gamma), _ptr(dres), _ptr(dx),
                                               _ptr(dx16), _ptr(part), rows, T, d, _stream_handle(stream)))
    return dx, dx16, part


def layernorm_bwd(dy, x, mean, rstd, gamma, dres, want_bf16=True, stream=None):
    T, d = x.shape
    dx = torch.empty(T, d, dtype=torch.float32, device="cuda")
    dx16 = torch.empty(T, d, dtype=torch.bfloat16, device="cuda") if want_bf16 else None
    part = torch.empty(((T + 7) // 8) * 3 * d, dtype=torch.float32, device="cuda")
    dg, db, dbias = (torch.empty(d, dtype=torch.float32, device="cuda") for _ in range(3))
    _check(_lib.lib().rv_k_layernorm_bwd(_ptr(dy), _ptr(x), _ptr(mean), _ptr(rstd), _ptr(gamma), _ptr(dres),
                                         _ptr(dx), _ptr(dx16), _ptr(part), _ptr(dg), _ptr(db), _ptr(dbias), T, d,
                                         _stream_handle(stream)))
    return dx, dx16, dg, db, dbias


def attention_fwd(qkv, mb, S, d, H, stream=None):
    out = torch.empty(mb * S, d, dtype=torch.bfloat16, device="cuda")
    lse2 = torch.empty(mb * H * S, dtype=torch.float32, device="cuda")
    _check(_lib.lib().rv_k_attention_fwd(_ptr(qkv), _ptr(out), _ptr(lse2), mb, S, d, H, _stream_handle(stream)))
    return out, lse2


def attention_bwd(qkv, out, dout, lse2, mb, S, d, H, stream=None):
    dqkv = torch.full((mb * S, 3 * d), float("nan"), dtype=torch.bfloat16, device="cuda")
    scratch = torch.empty(mb * H * S, dtype=torch.float32, device="cuda")
    _check(_lib.lib().rv_k_attention_bwd(_ptr(qkv), _ptr(out), _ptr(dout), _ptr(lse2), _ptr(scratch), _ptr(dqkv),
                                         mb, S, d, H, _stream_handle(stream)))
    return dqkv


def attention_bwd_static(qkv, out, dout, lse2, dqkv, mb, S, d, H, stream=None):
    """rv_k_attention_bwd_static: dqkv is the caller's output; nothing is allocated here or in the library."""
    _check(_lib.lib().rv_k_attention_bwd_static(_ptr(qkv), _ptr(out), _ptr(dout), _ptr(lse2), _ptr(dqkv), mb, S, d,
                                                H, _stream_handle(stream)))
    return dqkv


def _tokens(t, B, S, cols):
    """bf16 [B, S, cols], sequences one behind the other; the pitch of a token's row."""
    assert t.is_cuda and t.dtype is torch.bfloat16 and t.shape == (B, S, cols), (t.dtype, tuple(t.shape), (B, S, cols))
    per_sequence, per_token, per_column = t.stride()
    ld = per_token if S > 1 else per_sequence if B > 1 else cols
    assert per_column == 1 and (B == 1 or per_sequence == S * ld), "tokens one pitch apart, columns neighbours: strides %s" % (t.stride(),)
    return ld


def _cross_sizes(q, k, n_heads, n_kv_heads):
    B, Sq, cols = q.shape
    assert n_heads >= 1 and cols % n_heads == 0, (cols, n_heads)
    return B, Sq, k.shape[1], n_heads, n_kv_heads, cols // n_heads


@lru_cache(maxsize=256)
def _cross_work(sizes, backward):
    n = ctypes.c_size_t(0)
    _check(_lib.lib().rv_k_cross_attention_work(*sizes, backward, ctypes.byref(n)))
    return n.value


def cross_attention_fwd(q, k, v, n_heads, n_kv_heads, klen=None, out=None, stream=None):
    """rv_k_cross_attention_fwd: q bf16 [B, Sq, n_heads * d_head], k and v bf16 [B, Sk, n_kv_heads * d_head] (columns of a wider matrix
    or not), klen int32 [B] or None -> (out like q, lse2 fp32 [B, n_heads, Sq])."""
    sizes = B, Sq, Sk, H, Hkv, dh = _cross_sizes(q, k, n_heads, n_kv_heads)
    stream, context = _on(stream, q, k, v, klen, out)
    with context:
        out = torch.empty(B, Sq, H * dh, dtype=torch.bfloat16, device=q.device) if out is None else out
        lse2 = torch.empty(B, H, Sq, dtype=torch.float32, device=q.device)
        n = _cross_work(sizes, 0)
        work = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
        _check(_lib.lib().rv_k_cross_attention_fwd(
            _ptr(q), _tokens(q, B, Sq, H * dh), _ptr(k), _tokens(k, B, Sk, Hkv * dh), _ptr(v), _tokens(v, B, Sk, Hkv * dh),
            _ptr(_flat(klen, torch.int32, (B,)) if klen is not None else None), _ptr(out), _tokens(out, B, Sq, H * dh), _ptr(lse2), *sizes,
            _ptr(work), n, _stream_handle(stream)))
    return out, lse2


def cross_attention_bwd(q, k, v, out, dout, lse2, n_heads, n_kv_heads, klen=None, dq=None, dk=None, dv=None, stream=None):
    """rv_k_cross_attention_bwd: (dq, dk, dv) of the above; out and lse2 are the forward's."""
    sizes = B, Sq, Sk, H, Hkv, dh = _cross_sizes(q, k, n_heads, n_kv_heads)
    stream, context = _on(stream, q, k, v, klen, out, dout, lse2, dq, dk, dv)
    with context:
        dq, dk, dv = (torch.empty(t.shape, dtype=torch.bfloat16, device=q.device) if g is None else g for g, t in ((dq, q), (dk, k), (dv, v)))
        n = _cross_work(sizes, 1)
        work = torch.empty(n, dtype=torch.uint8, device=q.device)
        _check(_lib.lib().rv_k_cross_attention_bwd(
            _ptr(q), _tokens(q, B, Sq, H * dh), _ptr(k), _tokens(k, B, Sk, Hkv * dh), _ptr(v), _tokens(v, B, Sk, Hkv * dh),
            _ptr(_flat(klen, torch.int32, (B,)) if klen is not None else None), _ptr(out), _tokens(out, B, Sq, H * dh),
            _ptr(dout), _tokens(dout, B, Sq, H * dh), _ptr(_flat(lse2, torch.float32, (B, H, Sq))), _ptr(dq), _tokens(dq, B, Sq, H * dh),
            _ptr(dk), _tokens(dk, B, Sk, Hkv * dh), _ptr(dv), _tokens(dv, B, Sk, Hkv * dh), *sizes, _ptr(work), n, _stream_handle(stream)))
    return dq, dk, dv


_HERE = nullcontext()


def _handle(stream, first, *others):
    """As _on, for calls that take less time than it does: (the stream's handle, the context for memory)."""
    index = first.get_device()
    assert index >= 0, first.device
    for t in others:
        assert t is None or t.get_device() == index, "tensors of several devices: %s, %s" % (first.device, t.device)
    if stream is None:
        if index == torch.cuda.current_device():
            return torch._C._cuda_getCurrentRawStream(index), _HERE
        stream = torch.cuda.current_stream(index)
    assert stream.device_index == index, "a stream of %s for tensors of %s" % (stream.device, first.device)
    return stream.cuda_stream, torch.cuda.stream(stream)


def _address(t, dtype, shape):
    """Of a small tensor without gaps; 0 for None."""
    if t is None:
        return 0
    assert t.dtype is dtype and t.shape == shape and t.is_contiguous(), (t.dtype, tuple(t.shape), shape)
    return t.data_ptr()


def _matrix(t, B, S, cols):
    """(address, pitch); of None zeros."""
    return (0, 0) if t is None else (t.data_ptr(), _tokens(t, B, S, cols))


def _c_int(x):
    """A number of which any larger one means the same: ctypes would keep its low 32 bits, and struct refuse it."""
    return max(-1, min(x, 2 ** 31 - 1))


ROT_LAYOUT = {"half": 0, "pairs": 1}
FREQ_RULE = {"plain": 0, "linear": 1, "base": 2, "parts": 3}
# rv_rotary_desc as C lays it out: one call of pack() is a third of the time of filling in a ctypes structure
_ROTARY_DESC = struct.Struct("@7i2f6P" + "Pq" * 6 + "2i" + "Pq" * 4 + "3PNP")
assert _ROTARY_DESC.size == ctypes.sizeof(_lib.RotaryDesc)
_NONE = (0, 0)


def rotary_frequencies(rot, base=10000.0, rule="plain", factor=1.0, context=0.0, low=1.0, high=32.0):
    """rv_k_rotary_frequencies: (fp64 [rot / 2] in host memory, amplitude)."""
    freq, amplitude = torch.empty(max(1, rot // 2), dtype=torch.float64), ctypes.c_float(0.0)
    _check(_lib.lib().rv_k_rotary_frequencies(rot, base, FREQ_RULE[rule], factor, context, low, high, freq.data_ptr(), ctypes.byref(amplitude)))
    return freq, amplitude.value


def _rotary_sizes(q, k, n_heads, n_kv_heads):
    """(B, S, d_head) of any two of a call's matrices [B, S, columns], one of which may be None."""
    assert (q is None) == (n_heads == 0) and (k is None) == (n_kv_heads == 0), (n_heads, n_kv_heads)
    B, S, cols = (q if q is not None else k).shape
    heads = n_heads or n_kv_heads
    assert heads >= 1 and cols % heads == 0, (cols, heads)
    return B, S, cols // heads


def _rotary_head(B, S, n_heads, n_kv_heads, dh, freq, layout, amplitude, gamma_q, gamma_k, eps, pos, start, length):
    """What a description of either direction begins with."""
    half = 0 if freq is None else freq.numel()
    return (B, S, n_heads, n_kv_heads, dh, 2 * half, ROT_LAYOUT[layout], amplitude, eps, _address(freq, torch.float64, (half,)), _address(pos, torch.int32, (B, S)),
            _address(start, torch.int32, (B,)), _address(length, torch.int32, (B,)), _address(gamma_q, torch.bfloat16, (dh,)),
            _address(gamma_k, torch.bfloat16, (dh,)))


def rotary_fwd(q, k, freq, n_heads, n_kv_heads, *, v=None, layout="half", amplitude=1.0, gamma_q=None, gamma_k=None, eps=1e-6, pos=None, start=None,
               length=None, q_out=None, k_out=None, v_out=None, cache=None, sinks=0, stream=None):
    """rv_k_rotary_fwd: q bf16 [B, S, n_heads * d_head], k and v bf16 [B, S, n_kv_heads * d_head] (columns of a wider matrix or not; q or k None with no
    heads of it), freq device fp64 [rot / 2] or None, start and length int32 [B], pos int32 [B, S] -> (q_out, k_out) or, with v, (q_out, k_out, v_out).
    cache: (keys, values) bf16 [B, rows, n_kv_heads * d_head] in place of k_out and v_out (values None without v)."""
    B, S, dh = _rotary_sizes(q, k, n_heads, n_kv_heads)
    rows, qcols, kcols = 0, n_heads * dh, n_kv_heads * dh
    if cache is not None:
        assert k is not None and k_out is None and v_out is None
        k_out, v_out = cache
        rows = k_out.shape[1]
        assert (v is None) == (v_out is None)
    handle, context = _handle(stream, q if q is not None else k, k, freq, v, gamma_q, gamma_k, pos, start, length, q_out, k_out, v_out)
    with context:
        if q_out is None and q is not None:
            q_out = q.new_empty(B, S, qcols)
        if k_out is None and k is not None:
            k_out = k.new_empty(B, S, kcols)
        if v_out is None and v is not None:
            v_out = v.new_empty(B, S, kcols)
        _check(_lib.lib().rv_k_rotary_fwd(_ROTARY_DESC.pack(
            *_rotary_head(B, S, n_heads, n_kv_heads, dh, freq, layout, amplitude, gamma_q, gamma_k, eps, pos, start, length), *_matrix(q, B, S, qcols),
            *_matrix(k, B, S, kcols), *_matrix(v, B, S, kcols), *_matrix(q_out, B, S, qcols), *_matrix(k_out, B, rows or S, kcols),
            *_matrix(v_out, B, rows or S, kcols), rows, _c_int(sinks), *_NONE, *_NONE, *_NONE, *_NONE, 0, 0, 0, 0, handle)))
    return (q_out, k_out) if v is None else (q_out, k_out, v_out)


@lru_cache(maxsize=256)
def _rotary_work(B, S, n_heads, n_kv_heads, dh):
    n = ctypes.c_size_t(0)
    _check(_lib.lib().rv_k_rotary_work(B, S, n_heads, n_kv_heads, dh, ctypes.byref(n)))
    return n.value


def rotary_bwd(dq_out, dk_out, freq, n_heads, n_kv_heads, *, q=None, k=None, layout="half", amplitude=1.0, gamma_q=None, gamma_k=None, eps=1e-6, pos=None,
               start=None, length=None, dq=None, dk=None, weights=True, stream=None):
    """rv_k_rotary_bwd: (dq, dk, dgamma_q, dgamma_k) of the above; q and k, the forward's inputs, with norms only.  weights False: no dgamma."""
    B, S, dh = _rotary_sizes(dq_out, dk_out, n_heads, n_kv_heads)
    qcols, kcols = n_heads * dh, n_kv_heads * dh
    like = dq_out if dq_out is not None else dk_out
    handle, context = _handle(stream, like, dk_out, freq, q, k, gamma_q, gamma_k, pos, start, length, dq, dk)
    with context:
        if dq is None and dq_out is not None:
            dq = like.new_empty(B, S, qcols)
        if dk is None and dk_out is not None:
            dk = like.new_empty(B, S, kcols)
        n, work, dgamma_q, dgamma_k = 0, None, None, None
        if weights and (gamma_q is not None or gamma_k is not None):
            n = _rotary_work(B, S, n_heads, n_kv_heads, dh)
            work = like.new_empty(n, dtype=torch.uint8)
            dgamma_q, dgamma_k = (like.new_empty(dh, dtype=torch.float32) if g is not None else None for g in (gamma_q, gamma_k))
        address = lambda t: t.data_ptr() if t is not None else 0  # noqa: E731
        _check(_lib.lib().rv_k_rotary_bwd(_ROTARY_DESC.pack(
            *_rotary_head(B, S, n_heads, n_kv_heads, dh, freq, layout, amplitude, gamma_q, gamma_k, eps, pos, start, length), *_matrix(q, B, S, qcols),
            *_matrix(k, B, S, kcols), *_NONE, *_NONE, *_NONE, *_NONE, 0, 0, *_matrix(dq_out, B, S, qcols), *_matrix(dk_out, B, S, kcols), *_matrix(dq, B, S, qcols),
            *_matrix(dk, B, S, kcols), address(dgamma_q), address(dgamma_k), address(work), n, handle)))
    return dq, dk, dgamma_q, dgamma_k


@lru_cache(maxsize=256)
def _window_work(sizes, backward):
    n = ctypes.c_size_t(0)
    _check(_lib.lib().rv_k_window_attention_work(*sizes, backward, ctypes.byref(n)))
    return n.value


def window_attention_fwd(q, k, v, n_heads, n_kv_heads, window, sinks=0, start=None, length=None, out=None, stream=None):
    """rv_k_window_attention_fwd: q bf16 [B, Sq, n_heads * d_head], k and v bf16 [B, Sk, n_kv_heads * d_head] (columns of a wider matrix or not), start and
    length int32 [B] or None -> (out like q, lse2 fp32 [B, n_heads, Sq])."""
    B, Sq, Sk, H, Hkv, dh = _cross_sizes(q, k, n_heads, n_kv_heads)
    cols, kcols, sizes = H * dh, Hkv * dh, (B, Sq, Sk, H, Hkv, dh, _c_int(window), _c_int(sinks))
    handle, context = _handle(stream, q, k, v, start, length, out)
    with context:
        if out is None:
            out = q.new_empty(B, Sq, cols)
        lse2 = q.new_empty((B, H, Sq), dtype=torch.float32)
        n = _window_work(sizes, 0)
        work = q.new_empty(n, dtype=torch.uint8).data_ptr() if n else 0
        _check(_lib.lib().rv_k_window_attention_fwd(
            *_matrix(q, B, Sq, cols), *_matrix(k, B, Sk, kcols), *_matrix(v, B, Sk, kcols), _address(start, torch.int32, (B,)),
            _address(length, torch.int32, (B,)), *_matrix(out, B, Sq, cols), lse2.data_ptr(), *sizes, work, n, handle))
    return out, lse2


def window_attention_bwd(q, k, v, out, dout, lse2, n_heads, n_kv_heads, window, sinks=0, length=None, dq=None, dk=None, dv=None, stream=None):
    """rv_k_window_attention_bwd: (dq, dk, dv) of the above without start; out and lse2 are the forward's."""
    B, S, Sk, H, Hkv, dh = _cross_sizes(q, k, n_heads, n_kv_heads)
    assert S == Sk, (S, Sk)
    cols, kcols, window, sinks = H * dh, Hkv * dh, _c_int(window), _c_int(sinks)
    handle, context = _handle(stream, q, k, v, length, out, dout, lse2, dq, dk, dv)
    with context:
        dq = q.new_empty(B, S, cols) if dq is None else dq
        dk = q.new_empty(B, S, kcols) if dk is None else dk
        dv = q.new_empty(B, S, kcols) if dv is None else dv
        n = _window_work((B, S, S, H, Hkv, dh, window, sinks), 1)
        work = q.new_empty(n, dtype=torch.uint8)
        _check(_lib.lib().rv_k_window_attention_bwd(
            *_matrix(q, B, S, cols), *_matrix(k, B, S, kcols), *_matrix(v, B, S, kcols), _address(length, torch.int32, (B,)), *_matrix(out, B, S, cols),
            *_matrix(dout, B, S, cols), _address(lse2, torch.float32, (B, H, S)), *_matrix(dq, B, S, cols), *_matrix(dk, B, S, kcols),
            *_matrix(dv, B, S, kcols), B, S, H, Hkv, dh, window, sinks, work.data_ptr(), n, handle))
    return dq, dk, dv
