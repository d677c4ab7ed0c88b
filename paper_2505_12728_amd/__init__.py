"""SpecFLASH draft-verify hot path on MI355X: Python binding of libspecflash.

The three entry points mirror the C ABI in include/specflash.h and only
marshal arguments: every step of the computation runs in the HIP kernels of
libspecflash.so (built by ``paper_2505_12728_amd.build``).  torch supplies
device memory and the current HIP stream.  There is no fallback: if the
library is missing or the tensors are not on the GPU, the calls raise.

    sd_latent_compress   Sec. 3.2, Eq. 3 (learned queries attend over F_V)
    sd_verify_attention  Sec. 3.1 (one parallel pass over the K drafts)
    sd_spec_accept       Sec. 3.1 / 3.3 acceptance; greedy for Sec. 4.2
    sd_lm_head_probs     Sec. 3.1 / 3.3, Algorithm 1: LM head + softmax(z / tau)
    sd_sample_tokens     Algorithm 1: drafts drawn from their distributions
    sd_rope              rotary positions with one to four axes
    sd_kv_append         new rows rotated and written into the target's cache
    sd_verify_shared     verification attention of sequences that share prefixes
"""

import ctypes
import math
import os

__all__ = [
    "SD_OK", "SD_ERR_INVALID_ARG", "SD_ERR_UNSUPPORTED", "SD_ERR_WORKSPACE", "SD_ERR_HIP",
    "SD_F32", "SD_BF16", "SD_ACCEPT_GREEDY", "SD_ACCEPT_SAMPLED",
    "SDError", "library", "library_path",
    "sd_status_string", "sd_version",
    "sd_latent_compress_workspace_size", "sd_latent_compress",
    "sd_verify_workspace_size", "sd_verify_attention",
    "sd_spec_accept_workspace_size", "sd_spec_accept", "sd_spec_accept_noalloc",
    "sd_lm_head_workspace_size", "sd_lm_head_probs",
    "sd_sample_workspace_size", "sd_sample_tokens",
    "sd_spec_accept_logits_workspace_size", "sd_spec_accept_logits", "sd_philox_uniforms",
    "sd_linear_workspace_size", "sd_linear",
    "sd_semi_ar_layer_workspace_size", "sd_semi_ar_layer",
    "sd_semi_ar_draft_workspace_size", "sd_semi_ar_draft",
    "sd_linear_q8", "sd_semi_ar_layer_q8", "sd_avg_pool_compress",
    "sd_latent_compress_q8_workspace_size", "sd_latent_compress_q8",
    "SD_ROPE_RUNNING", "SD_ROPE_PER_AXIS", "sd_rope", "sd_kv_append",
    "sd_verify_shared_workspace_size", "sd_verify_shared",
]

SD_OK, SD_ERR_INVALID_ARG, SD_ERR_UNSUPPORTED, SD_ERR_WORKSPACE, SD_ERR_HIP = 0, 1, 2, 3, 4
SD_F32, SD_BF16 = 0, 1
SD_ACCEPT_GREEDY, SD_ACCEPT_SAMPLED = 0, 1
SD_ROPE_RUNNING, SD_ROPE_PER_AXIS = 0, 1

_HERE = os.path.dirname(os.path.abspath(__file__))
library_path = os.path.join(_HERE, "libspecflash.so")
_lib = None

_c = ctypes
_vp, _sz, _i, _f, _i64 = _c.c_void_p, _c.c_size_t, _c.c_int, _c.c_float, _c.c_int64
_SIGNATURES = {
    "sd_status_string": (_c.c_char_p, [_i]),
    "sd_version": (_i, []),
    "sd_latent_compress_workspace_size": (_sz, [_i, _i, _i, _i, _i, _i]),
    "sd_latent_compress": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _f, _i, _vp, _sz, _vp]),
    "sd_verify_workspace_size": (_sz, [_i, _i, _i, _i, _i, _i, _i]),
    "sd_verify_attention": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _vp, _vp,
                                 _i, _i, _i, _i, _i, _f, _i, _vp, _sz, _vp]),
    "sd_spec_accept_workspace_size": (_sz, [_i, _i, _i, _i]),
    "sd_spec_accept": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _vp, _sz, _vp]),
    "sd_spec_accept_noalloc": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _vp]),
    "sd_spec_accept_logits_workspace_size": (_sz, [_i, _i, _i, _i]),
    "sd_spec_accept_logits": (_i, [_vp, _vp, _vp, ctypes.c_uint64, ctypes.c_uint64, ctypes.c_float,
                                   _vp, _vp, _i, _i, _i, _i, _i, _vp, _sz, _vp]),
    "sd_philox_uniforms": (_i, [ctypes.c_uint64, ctypes.c_uint64, _vp, _i, _i, _vp]),
    "sd_lm_head_workspace_size": (_sz, [_i, _i, _i, _i]),
    "sd_lm_head_probs": (_i, [_vp, _vp, _vp, _i, _i, _i, _f, _i, _vp, _sz, _vp]),
    "sd_sample_workspace_size": (_sz, [_i, _i]),
    "sd_sample_tokens": (_i, [_vp, _vp, _vp, _i, _i, _vp, _sz, _vp]),
    "sd_linear_workspace_size": (_sz, [_i, _i, _i]),
    "sd_linear": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _vp, _sz, _vp]),
    "sd_semi_ar_layer_workspace_size": (_sz, [_i, _i, _i, _i, _i, _i, _i]),
    "sd_semi_ar_layer": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                              _i, _i, _i, _i, _i, _i, _i, _f, _f, _vp, _sz, _vp]),
    "sd_semi_ar_draft_workspace_size": (_sz, [_i] * 10),
    "sd_linear_q8": (_i, [_vp] * 6 + [_i, _i, _i, _vp, _sz, _vp]),
    "sd_avg_pool_compress": (_i, [_vp, _vp, _i, _i, _i, _i, _i, _vp]),
    "sd_latent_compress_q8_workspace_size": (_sz, [_i, _i, _i, _i, _i]),
    "sd_latent_compress_q8": (_i, [_vp] * 5 + [_i] * 5 + [_f, _vp, _sz, _vp]),
    "sd_semi_ar_layer_q8": (_i, [_vp] * 18 + [_i] * 7 + [_f, _f, _vp, _sz, _vp]),
    "sd_semi_ar_draft": (_i, [_vp] * 18 + [_i] * 10 + [_f, _f, _f, _vp, _sz, _vp]),
    "sd_rope": (_i, [_vp, _i64, _vp, _vp, _i64, _i, _i, _i, _i, _vp, _f, _i, _i, _i, _vp]),
    "sd_kv_append": (_i, [_vp, _i64] * 3 + [_vp] * 6 + [_i, _i, _i, _vp] + [_i] * 6 + [_vp, _f, _i, _i, _i, _vp]),
    "sd_verify_shared_workspace_size": (_sz, [_i] * 9),
    "sd_verify_shared": (_i, [_vp] * 5 + [_i] * 3 + [_vp] * 4 + [_i] * 3 + [_vp] * 3 + [_i] * 6
                         + [_f, _i, _i, _vp, _sz, _vp]),
}


class SDError(RuntimeError):
    """A non-zero sd_status returned by the library."""

    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {sd_status_string(status)}")


def library():
    """Load libspecflash.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(library_path):
            raise RuntimeError(
                f"{library_path} is missing: build it with `python -m paper_2505_12728_amd.build`")
        lib = ctypes.CDLL(library_path)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def sd_status_string(status):
    return library().sd_status_string(int(status)).decode()


def sd_version():
    return library().sd_version()


# ----------------------------------------------------------------- helpers

# A call's host time is part of every small operation (acceptance of one
# sequence: 12.2 us of host time around a 6.9 us kernel before, 8.9 us now),
# so the checks below take one pass over the tensor's properties and leave
# the messages to a second one, pointers go to ctypes as plain integers, and
# the current stream is read without building a torch Stream object.

_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _dtype_code(t):
    torch = _torch()
    if t.dtype == torch.float32:
        return SD_F32
    if t.dtype == torch.bfloat16:
        return SD_BF16
    raise TypeError(f"unsupported dtype {t.dtype}: use float32 or bfloat16")


def _check(t, name, dtype=None, ndim=None):
    if (t.is_cuda and t.is_contiguous() and (dtype is None or t.dtype == dtype)
            and (ndim is None or t.dim() == ndim)):
        return
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dimensions, got {t.dim()}")


def _out(t, name, shape, dtype, device):
    """A caller-supplied output (or workspace) must be a contiguous tensor of
    exactly the expected shape and dtype on the inputs' device: the kernels
    write its whole extent, so a short buffer would be overrun on the device."""
    _check(t, name, dtype)
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}, got {t.device}")
    return t


def _same_device(name, t, device):
    if t is not None and t.device != device:
        raise ValueError(f"{name} must be on {device}, got {t.device}")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _on_current(names, *tensors):
    """The library launches on the current device: every tensor (None: left
    out) lies there.  One comparison each; the messages come afterwards."""
    c = _torch()._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != c:
            name = names.split()[[x is t for x in tensors].index(True)]
            if not t.is_cuda:
                raise ValueError(f"{name} must be a GPU tensor")
            raise ValueError(f"{name} must be on cuda:{c}, the current device, got {t.device}")


def _dense(t, name, dtype, ndim):
    if t.dtype == dtype and t.dim() == ndim and t.is_contiguous():
        return
    _check(t, name, dtype, ndim)


def _pages(num_pages, pool):
    """Pages a call may use: all of the pool's, or fewer of them."""
    if num_pages is None:
        return pool.shape[0]
    if not 1 <= num_pages <= pool.shape[0]:
        raise ValueError(f"num_pages must be 1 .. {pool.shape[0]}, the pages of the pool")
    return num_pages


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    c = _torch()._C
    return c._cuda_getCurrentRawStream(c._cuda_getDevice())


def _workspace(nbytes, device, given):
    if nbytes == 0:
        return None, 0
    if given is not None:
        _check(given, "workspace")
        _same_device("workspace", given, device)
        return given, given.numel() * given.element_size()
    torch = _torch()
    # zero-filled: some entry points keep arrival counters in the workspace
    # that must start at zero (every call returns them to zero)
    return torch.zeros(nbytes, dtype=torch.uint8, device=device), nbytes


def _empty(shape, strides, dtype, device, stream):
    """Memory for a call on `stream`: a given stream's own, so that the
    allocator reuses it behind that stream's work.  Plain tuples: 1.3 us, where
    torch.empty takes 1.7, and 2.3 from a torch.Size."""
    torch = _torch()
    if stream is None:
        return torch.empty_strided(shape, strides, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty_strided(shape, strides, dtype=dtype, device=device)


def _scratch(nbytes, device, given, stream):
    """_workspace for calls that keep no counters in it: left as allocated."""
    if given is not None or nbytes == 0:
        return _workspace(nbytes, device, given)
    return _empty((nbytes,), (1,), _torch().uint8, device, stream), nbytes


def _raise(status, where):
    if status != SD_OK:
        raise SDError(status, where)


# ------------------------------------------------------------- compression

def sd_latent_compress_workspace_size(B, N, C, d, num_heads, dtype):
    return library().sd_latent_compress_workspace_size(B, N, C, d, num_heads, dtype)


def sd_latent_compress(latents, feats, num_heads=1, scale=1.0, out=None, workspace=None,
                       stream=None):
    """Eq. 3 per head slice: latents [C, d], feats [B, N, d] -> out [B, C, d] fp32."""
    torch = _torch()
    _check(latents, "latents", ndim=2)
    _check(feats, "feats", dtype=latents.dtype, ndim=3)
    C, d = latents.shape
    B, N, d2 = feats.shape
    if d2 != d:
        raise ValueError("latents and feats disagree on the feature width")
    dt = _dtype_code(latents)
    _same_device("feats", feats, latents.device)
    if out is None:
        out = torch.empty((B, C, d), dtype=torch.float32, device=feats.device)
    _out(out, "out", (B, C, d), torch.float32, feats.device)
    ws_bytes = sd_latent_compress_workspace_size(B, N, C, d, num_heads, dt)
    ws, ws_len = _workspace(ws_bytes, feats.device, workspace)
    st = library().sd_latent_compress(_ptr(latents), _ptr(feats), _ptr(out), B, N, C, d,
                                      num_heads, float(scale), dt, _ptr(ws), ws_len,
                                      _stream(stream))
    _raise(st, "sd_latent_compress")
    return out


def sd_latent_compress_q8_workspace_size(B, N, C, d, num_heads):
    return library().sd_latent_compress_q8_workspace_size(B, N, C, d, num_heads)


def sd_latent_compress_q8(latents_q, latent_exp, feats_q, feat_exp, num_heads=1, scale=1.0, out=None,
                          workspace=None, stream=None):
    """Eq. 3 on int8 rows with power-of-two row scales: latents_q [C, d] int8
    with latent_exp [C] int8, feats_q [B, N, d] int8 with feat_exp [B, N]
    int8 (row r stands for q[r] * 2^e[r]).  Returns out [B, C, d] fp32."""
    torch = _torch()
    _check(latents_q, "latents_q", dtype=torch.int8, ndim=2)
    _check(feats_q, "feats_q", dtype=torch.int8, ndim=3)
    _check(latent_exp, "latent_exp", dtype=torch.int8, ndim=1)
    _check(feat_exp, "feat_exp", dtype=torch.int8, ndim=2)
    C, d = latents_q.shape
    B, N, d2 = feats_q.shape
    if d2 != d or latent_exp.shape[0] != C or tuple(feat_exp.shape) != (B, N):
        raise ValueError("latents_q [C, d], latent_exp [C], feats_q [B, N, d], feat_exp [B, N] expected")
    dev = feats_q.device
    for name, t in (("latents_q", latents_q), ("latent_exp", latent_exp), ("feat_exp", feat_exp)):
        _same_device(name, t, dev)
    if out is None:
        out = torch.empty((B, C, d), dtype=torch.float32, device=dev)
    _out(out, "out", (B, C, d), torch.float32, dev)
    ws_bytes = sd_latent_compress_q8_workspace_size(B, N, C, d, num_heads)
    ws, ws_len = _workspace(ws_bytes, dev, workspace)
    st = library().sd_latent_compress_q8(_ptr(latents_q), _ptr(latent_exp), _ptr(feats_q), _ptr(feat_exp),
                                         _ptr(out), B, N, C, d, num_heads, float(scale), _ptr(ws), ws_len,
                                         _stream(stream))
    _raise(st, "sd_latent_compress_q8")
    return out


# ------------------------------------------------------------ verification

def sd_verify_workspace_size(B, k, Hq, Hkv, D, capacity, dtype):
    return library().sd_verify_workspace_size(B, k, Hq, Hkv, D, capacity, dtype)


def sd_verify_attention(q, k_cache, v_cache, kv_len, scale=None, page_table=None,
                        num_pages=None, out=None, lse=True, workspace=None, stream=None):
    """Attention of the k block queries over the cache (causal inside the block).

    q [B, k, Hq, D]; caches [B, Lmax, Hkv, D], or page pools [P, Hkv, 16, D]
    with page_table [B, max_pages] int32; kv_len [B] int32 (block included).
    Returns (out [B, k, Hq, D] fp32, lse [B, k, Hq] fp32 or None).
    ``scale`` multiplies q . k; the paper names no scale, and None passes the
    standard attention scale 1 / sqrt(D) to the library explicitly (the C
    entry point itself takes the scale as a required argument).
    """
    torch = _torch()
    _check(q, "q", ndim=4)
    _check(k_cache, "k_cache", dtype=q.dtype, ndim=4)
    _check(v_cache, "v_cache", dtype=q.dtype, ndim=4)
    _check(kv_len, "kv_len", dtype=torch.int32, ndim=1)
    B, k, Hq, D = q.shape
    if tuple(k_cache.shape) != tuple(v_cache.shape):
        raise ValueError("k_cache and v_cache must have the same shape")
    if kv_len.shape[0] != B:
        raise ValueError("kv_len needs one entry per sequence")
    dt = _dtype_code(q)
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if page_table is None:
        if k_cache.shape[0] != B or k_cache.shape[3] != D:
            raise ValueError("contiguous caches must be [B, Lmax, Hkv, D]")
        Lmax, Hkv = k_cache.shape[1], k_cache.shape[2]
        max_pages = num_pages_ = 0
        capacity = Lmax
    else:
        _check(page_table, "page_table", dtype=torch.int32, ndim=2)
        if k_cache.shape[2] != 16 or k_cache.shape[3] != D or page_table.shape[0] != B:
            raise ValueError("paged caches must be [P, Hkv, 16, D] with a [B, max_pages] table")
        Hkv = k_cache.shape[1]
        max_pages = page_table.shape[1]
        num_pages_ = k_cache.shape[0] if num_pages is None else num_pages
        Lmax = 0
        capacity = 16 * max_pages
    for name, t in (("k_cache", k_cache), ("v_cache", v_cache), ("kv_len", kv_len),
                    ("page_table", page_table)):
        _same_device(name, t, q.device)
    if out is None:
        out = torch.empty((B, k, Hq, D), dtype=torch.float32, device=q.device)
    _out(out, "out", (B, k, Hq, D), torch.float32, q.device)
    lse_t = None
    if lse is True:
        lse_t = torch.empty((B, k, Hq), dtype=torch.float32, device=q.device)
    elif lse is not None and lse is not False:
        lse_t = _out(lse, "lse", (B, k, Hq), torch.float32, q.device)
    ws_bytes = sd_verify_workspace_size(B, k, Hq, Hkv, D, capacity, dt)
    ws, ws_len = _workspace(ws_bytes, q.device, workspace)
    st = library().sd_verify_attention(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(kv_len),
                                       _ptr(page_table), max_pages, num_pages_, Lmax, _ptr(out),
                                       _ptr(lse_t), B, k, Hq, Hkv, D, float(scale), dt,
                                       _ptr(ws), ws_len, _stream(stream))
    _raise(st, "sd_verify_attention")
    return out, lse_t


# -------------------------------------------------------------- acceptance

def sd_spec_accept_workspace_size(B, k, V, mode):
    return library().sd_spec_accept_workspace_size(B, k, V, mode)


def sd_spec_accept(p, q, draft, u, mode=SD_ACCEPT_SAMPLED, n_accepted=None, tokens=None,
                   workspace=None, stream=None):
    """Speculative acceptance: p [B, k+1, V], q [B, k, V], draft [B, k] int32,
    u [B, k+1] fp32.  Returns (n_accepted [B] int32, tokens [B, k+1] int32)."""
    torch = _torch()
    _check(p, "p", dtype=torch.float32, ndim=3)
    _check(draft, "draft", dtype=torch.int32, ndim=2)
    B, kp1, V = p.shape
    k = kp1 - 1
    if tuple(draft.shape) != (B, k):
        raise ValueError("draft must be [B, k]")
    if mode == SD_ACCEPT_SAMPLED:
        _check(q, "q", dtype=torch.float32, ndim=3)
        _check(u, "u", dtype=torch.float32, ndim=2)
        if tuple(q.shape) != (B, k, V) or tuple(u.shape) != (B, k + 1):
            raise ValueError("q must be [B, k, V] and u [B, k+1]")
    for name, t in (("q", q if mode == SD_ACCEPT_SAMPLED else None), ("draft", draft),
                    ("u", u if mode == SD_ACCEPT_SAMPLED else None)):
        _same_device(name, t, p.device)
    if n_accepted is None:
        n_accepted = torch.empty((B,), dtype=torch.int32, device=p.device)
    if tokens is None:
        tokens = torch.empty((B, k + 1), dtype=torch.int32, device=p.device)
    _out(n_accepted, "n_accepted", (B,), torch.int32, p.device)
    _out(tokens, "tokens", (B, k + 1), torch.int32, p.device)
    ws_bytes = sd_spec_accept_workspace_size(B, k, V, mode)
    ws, ws_len = _workspace(ws_bytes, p.device, workspace)
    st = library().sd_spec_accept(_ptr(p), _ptr(q), _ptr(draft), _ptr(u), _ptr(n_accepted),
                                  _ptr(tokens), B, k, V, int(mode), _ptr(ws), ws_len,
                                  _stream(stream))
    _raise(st, "sd_spec_accept")
    return n_accepted, tokens


def sd_spec_accept_noalloc(p, q, draft, u, mode=SD_ACCEPT_SAMPLED, n_accepted=None, tokens=None,
                           stream=None):
    """sd_spec_accept with the library's fixed device scratch instead of a
    workspace (for callers that cannot allocate; pass n_accepted and tokens
    to allocate nothing here either).  Same arguments and results."""
    torch = _torch()
    _check(p, "p", dtype=torch.float32, ndim=3)
    _check(draft, "draft", dtype=torch.int32, ndim=2)
    B, kp1, V = p.shape
    k = kp1 - 1
    if tuple(draft.shape) != (B, k):
        raise ValueError("draft must be [B, k]")
    if mode == SD_ACCEPT_SAMPLED:
        _check(q, "q", dtype=torch.float32, ndim=3)
        _check(u, "u", dtype=torch.float32, ndim=2)
        if tuple(q.shape) != (B, k, V) or tuple(u.shape) != (B, k + 1):
            raise ValueError("q must be [B, k, V] and u [B, k+1]")
        _same_device("q", q, p.device)
        _same_device("u", u, p.device)
    _same_device("draft", draft, p.device)
    if n_accepted is None:
        n_accepted = torch.empty((B,), dtype=torch.int32, device=p.device)
    if tokens is None:
        tokens = torch.empty((B, k + 1), dtype=torch.int32, device=p.device)
    _out(n_accepted, "n_accepted", (B,), torch.int32, p.device)
    _out(tokens, "tokens", (B, k + 1), torch.int32, p.device)
    st = library().sd_spec_accept_noalloc(_ptr(p), _ptr(q), _ptr(draft), _ptr(u), _ptr(n_accepted),
                                          _ptr(tokens), B, k, V, int(mode), _stream(stream))
    _raise(st, "sd_spec_accept_noalloc")
    return n_accepted, tokens


def sd_spec_accept_logits_workspace_size(B, k, V, mode):
    return library().sd_spec_accept_logits_workspace_size(B, k, V, mode)


def sd_spec_accept_logits(target_logits, draft_logits, draft, seed, offset, temperature,
                          mode=SD_ACCEPT_SAMPLED, n_accepted=None, tokens=None, workspace=None,
                          stream=None):
    """Acceptance from logits: target_logits [B, k+1, V], draft_logits [B, k, V]
    (fp32 or bf16, same dtype), draft [B, k] int32; uniforms from Philox(seed,
    offset).  Returns (n_accepted [B] int32, tokens [B, k+1] int32)."""
    torch = _torch()
    _check(target_logits, "target_logits", ndim=3)
    _check(draft, "draft", dtype=torch.int32, ndim=2)
    B, kp1, V = target_logits.shape
    k = kp1 - 1
    if tuple(draft.shape) != (B, k):
        raise ValueError("draft must be [B, k]")
    if mode == SD_ACCEPT_SAMPLED:
        _check(draft_logits, "draft_logits", dtype=target_logits.dtype, ndim=3)
        if tuple(draft_logits.shape) != (B, k, V):
            raise ValueError("draft_logits must be [B, k, V]")
    dt = _dtype_code(target_logits)
    dev = target_logits.device
    _same_device("draft", draft, dev)
    if mode == SD_ACCEPT_SAMPLED:
        _same_device("draft_logits", draft_logits, dev)
    if n_accepted is None:
        n_accepted = torch.empty((B,), dtype=torch.int32, device=dev)
    if tokens is None:
        tokens = torch.empty((B, k + 1), dtype=torch.int32, device=dev)
    _out(n_accepted, "n_accepted", (B,), torch.int32, dev)
    _out(tokens, "tokens", (B, k + 1), torch.int32, dev)
    ws_bytes = sd_spec_accept_logits_workspace_size(B, k, V, mode)
    ws, ws_len = _workspace(ws_bytes, target_logits.device, workspace)
    st = library().sd_spec_accept_logits(_ptr(target_logits), _ptr(draft_logits), _ptr(draft),
                                         int(seed), int(offset), float(temperature),
                                         _ptr(n_accepted), _ptr(tokens), B, k, V, dt, int(mode),
                                         _ptr(ws), ws_len, _stream(stream))
    _raise(st, "sd_spec_accept_logits")
    return n_accepted, tokens


def sd_philox_uniforms(seed, offset, B, n, out=None, device=None, stream=None):
    """u [B, n] float32 on the device: the acceptance uniforms of (seed, offset)."""
    torch = _torch()
    if out is None:
        out = torch.empty((B, n), dtype=torch.float32, device=device or "cuda")
    _out(out, "out", (B, n), torch.float32, out.device)
    st = library().sd_philox_uniforms(int(seed), int(offset), _ptr(out), B, n, _stream(stream))
    _raise(st, "sd_philox_uniforms")
    return out


def sd_lm_head_workspace_size(R, d, V, dtype):
    return library().sd_lm_head_workspace_size(R, d, V, dtype)


def sd_lm_head_probs(hidden, weight, temperature, out=None, workspace=None, stream=None):
    """LM head + temperature softmax: hidden [R, d], weight [V, d] (bf16 or
    fp32, same dtype).  Returns probs [R, V] fp32 = softmax(hidden W^T / tau)."""
    torch = _torch()
    _check(hidden, "hidden", ndim=2)
    _check(weight, "weight", dtype=hidden.dtype, ndim=2)
    R, d = hidden.shape
    V = weight.shape[0]
    if weight.shape[1] != d:
        raise ValueError("weight must be [V, d] with the hidden width d")
    dt = _dtype_code(hidden)
    _same_device("weight", weight, hidden.device)
    if out is None:
        out = torch.empty((R, V), dtype=torch.float32, device=hidden.device)
    _out(out, "out", (R, V), torch.float32, hidden.device)
    ws_bytes = sd_lm_head_workspace_size(R, d, V, dt)
    ws, ws_len = _workspace(ws_bytes, hidden.device, workspace)
    st = library().sd_lm_head_probs(_ptr(hidden), _ptr(weight), _ptr(out), R, d, V,
                                    float(temperature), dt, _ptr(ws), ws_len, _stream(stream))
    _raise(st, "sd_lm_head_probs")
    return out


def sd_sample_workspace_size(R, V):
    return library().sd_sample_workspace_size(R, V)


def sd_sample_tokens(probs, u, out=None, workspace=None, stream=None):
    """T_r ~ Categorical(probs[r]) (exact fixed-point inverse CDF): probs [R, V]
    fp32, u [R] fp32.  Returns tokens [R] int32."""
    torch = _torch()
    _check(probs, "probs", dtype=torch.float32, ndim=2)
    _check(u, "u", dtype=torch.float32, ndim=1)
    R, V = probs.shape
    if u.shape[0] != R:
        raise ValueError("u must be [R]")
    _same_device("u", u, probs.device)
    if out is None:
        out = torch.empty((R,), dtype=torch.int32, device=probs.device)
    _out(out, "out", (R,), torch.int32, probs.device)
    ws_bytes = sd_sample_workspace_size(R, V)
    ws, ws_len = _workspace(ws_bytes, probs.device, workspace)
    st = library().sd_sample_tokens(_ptr(probs), _ptr(u), _ptr(out), R, V, _ptr(ws), ws_len,
                                    _stream(stream))
    _raise(st, "sd_sample_tokens")
    return out


def sd_linear_workspace_size(R, K, N):
    return library().sd_linear_workspace_size(R, K, N)


def sd_linear(x, w, bias=None, residual=None, out=None, workspace=None, stream=None):
    """y = x W^T (+ bias) (+ residual): x [R, K] bf16, w [N, K] bf16, bias [N]
    fp32, residual [R, N] fp32.  Returns y [R, N] fp32."""
    torch = _torch()
    _check(x, "x", dtype=torch.bfloat16, ndim=2)
    _check(w, "w", dtype=torch.bfloat16, ndim=2)
    R, K = x.shape
    N = w.shape[0]
    if w.shape[1] != K:
        raise ValueError("w must be [N, K] with the width K of x")
    if bias is not None:
        _check(bias, "bias", dtype=torch.float32, ndim=1)
        if bias.shape[0] != N:
            raise ValueError("bias must be [N]")
    if residual is not None:
        _check(residual, "residual", dtype=torch.float32, ndim=2)
        if tuple(residual.shape) != (R, N):
            raise ValueError("residual must be [R, N]")
    for name, t in (("w", w), ("bias", bias), ("residual", residual)):
        _same_device(name, t, x.device)
    if out is None:
        out = torch.empty((R, N), dtype=torch.float32, device=x.device)
    _out(out, "out", (R, N), torch.float32, x.device)
    ws_bytes = sd_linear_workspace_size(R, K, N)
    ws, ws_len = _workspace(ws_bytes, x.device, workspace)
    st = library().sd_linear(_ptr(x), _ptr(w), _ptr(bias), _ptr(residual), _ptr(out), R, K, N,
                             _ptr(ws), ws_len, _stream(stream))
    _raise(st, "sd_linear")
    return out


def sd_semi_ar_layer_workspace_size(B, r, d, hq, hkv, I, Lmax):
    return library().sd_semi_ar_layer_workspace_size(B, r, d, hq, hkv, I, Lmax)


SEMI_AR_WEIGHTS = ("fc_w", "fc_b", "ln1", "wqkv", "wo", "ln2", "wgu", "wdown")


def sd_semi_ar_layer(u, weights, k_cache, v_cache, pos, hq, hkv, eps, theta, out=None,
                     workspace=None, stream=None):
    """One draft step of the semi-autoregressive layer.  u [B, r, 2d] bf16;
    weights: dict of fc_w [d, 2d], wqkv [(hq + 2 hkv) D, d], wo [d, hq D],
    wgu [2I, d], wdown [d, I] (bf16) and fc_b, ln1, ln2 [d] (fp32); caches
    [B, Lmax, hkv, D] bf16 (updated in place at positions pos[b] ..
    pos[b] + r - 1); pos [B] int32.  Returns out [B, r, d] fp32."""
    torch = _torch()
    _check(u, "u", dtype=torch.bfloat16, ndim=3)
    B, r, d2 = u.shape
    d = d2 // 2
    for name in SEMI_AR_WEIGHTS:
        t = weights[name]
        _check(t, name, dtype=torch.float32 if name in ("fc_b", "ln1", "ln2") else torch.bfloat16)
    _check(k_cache, "k_cache", dtype=torch.bfloat16, ndim=4)
    _check(v_cache, "v_cache", dtype=torch.bfloat16, ndim=4)
    _check(pos, "pos", dtype=torch.int32, ndim=1)
    Lmax = k_cache.shape[1]
    I = weights["wdown"].shape[1]
    D = d // hq
    shapes = {"fc_w": (d, 2 * d), "fc_b": (d,), "ln1": (d,), "wqkv": ((hq + 2 * hkv) * D, d),
              "wo": (d, hq * D), "ln2": (d,), "wgu": (2 * I, d), "wdown": (d, I)}
    for name, shp in shapes.items():
        if tuple(weights[name].shape) != shp:
            raise ValueError(f"{name} must be {shp}, got {tuple(weights[name].shape)}")
    if tuple(k_cache.shape) != (B, Lmax, hkv, D) or tuple(v_cache.shape) != (B, Lmax, hkv, D):
        raise ValueError("caches must be [B, Lmax, hkv, d / hq]")
    if pos.shape[0] != B:
        raise ValueError("pos must be [B]")
    for name, t in [(n, weights[n]) for n in SEMI_AR_WEIGHTS] + [
            ("k_cache", k_cache), ("v_cache", v_cache), ("pos", pos)]:
        _same_device(name, t, u.device)
    if out is None:
        out = torch.empty((B, r, d), dtype=torch.float32, device=u.device)
    _out(out, "out", (B, r, d), torch.float32, u.device)
    ws_bytes = sd_semi_ar_layer_workspace_size(B, r, d, hq, hkv, I, Lmax)
    ws, ws_len = _workspace(ws_bytes, u.device, workspace)
    W = weights
    st = library().sd_semi_ar_layer(_ptr(u), _ptr(W["fc_w"]), _ptr(W["fc_b"]), _ptr(W["ln1"]),
                                    _ptr(W["wqkv"]), _ptr(W["wo"]), _ptr(W["ln2"]), _ptr(W["wgu"]),
                                    _ptr(W["wdown"]), _ptr(k_cache), _ptr(v_cache), _ptr(pos),
                                    _ptr(out), B, r, d, hq, hkv, I, Lmax, float(eps), float(theta),
                                    _ptr(ws), ws_len, _stream(stream))
    _raise(st, "sd_semi_ar_layer")
    return out


def sd_semi_ar_draft_workspace_size(B, r0, d, hq, hkv, I, Lmax, V, K, kp):
    return library().sd_semi_ar_draft_workspace_size(B, r0, d, hq, hkv, I, Lmax, V, K, kp)


def sd_semi_ar_draft(u0, weights, lm_w, emb, ph, k_cache, v_cache, pos, u, K, kp, hq, hkv, eps, theta,
                     temperature, tokens=None, q=None, workspace=None, stream=None):
    """K drafts in K / kp passes of the semi-AR layer.  u0 [B, r0, 2d] bf16
    (last kp rows placeholders); weights as for sd_semi_ar_layer; lm_w and
    emb [V, d] bf16; ph [2d] bf16; u [B, K] fp32 uniforms.  The caches are
    updated in place.  Returns (tokens [B, K] int32, q [B, K, V] fp32)."""
    torch = _torch()
    _check(u0, "u0", dtype=torch.bfloat16, ndim=3)
    B, r0, d2 = u0.shape
    d = d2 // 2
    _check(lm_w, "lm_w", dtype=torch.bfloat16, ndim=2)
    _check(emb, "emb", dtype=torch.bfloat16, ndim=2)
    _check(ph, "ph", dtype=torch.bfloat16, ndim=1)
    _check(u, "u", dtype=torch.float32, ndim=2)
    V = lm_w.shape[0]
    if lm_w.shape[1] != d or tuple(emb.shape) != (V, d) or ph.shape[0] != 2 * d:
        raise ValueError("lm_w and emb must be [V, d], ph [2d]")
    if tuple(u.shape) != (B, K):
        raise ValueError("u must be [B, K]")
    for name in SEMI_AR_WEIGHTS:
        _check(weights[name], name, dtype=torch.float32 if name in ("fc_b", "ln1", "ln2") else torch.bfloat16)
    _check(k_cache, "k_cache", dtype=torch.bfloat16, ndim=4)
    _check(v_cache, "v_cache", dtype=torch.bfloat16, ndim=4)
    _check(pos, "pos", dtype=torch.int32, ndim=1)
    Lmax = k_cache.shape[1]
    I = weights["wdown"].shape[1]
    D = d // hq
    shapes = {"fc_w": (d, 2 * d), "fc_b": (d,), "ln1": (d,), "wqkv": ((hq + 2 * hkv) * D, d),
              "wo": (d, hq * D), "ln2": (d,), "wgu": (2 * I, d), "wdown": (d, I)}
    for name, shp in shapes.items():
        if tuple(weights[name].shape) != shp:
            raise ValueError(f"{name} must be {shp}, got {tuple(weights[name].shape)}")
    if tuple(k_cache.shape) != (B, Lmax, hkv, D) or tuple(v_cache.shape) != (B, Lmax, hkv, D):
        raise ValueError("caches must be [B, Lmax, hkv, d / hq]")
    if pos.shape[0] != B:
        raise ValueError("pos must be [B]")
    for name, t in [(n, weights[n]) for n in SEMI_AR_WEIGHTS] + [
            ("lm_w", lm_w), ("emb", emb), ("ph", ph), ("k_cache", k_cache),
            ("v_cache", v_cache), ("pos", pos), ("u", u)]:
        _same_device(name, t, u0.device)
    if tokens is None:
        tokens = torch.empty((B, K), dtype=torch.int32, device=u0.device)
    if q is None:
        q = torch.empty((B, K, V), dtype=torch.float32, device=u0.device)
    _out(tokens, "tokens", (B, K), torch.int32, u0.device)
    _out(q, "q", (B, K, V), torch.float32, u0.device)
    ws_bytes = sd_semi_ar_draft_workspace_size(B, r0, d, hq, hkv, I, Lmax, V, K, kp)
    ws, ws_len = _workspace(ws_bytes, u0.device, workspace)
    W = weights
    st = library().sd_semi_ar_draft(_ptr(u0), _ptr(W["fc_w"]), _ptr(W["fc_b"]), _ptr(W["ln1"]),
                                    _ptr(W["wqkv"]), _ptr(W["wo"]), _ptr(W["ln2"]), _ptr(W["wgu"]),
                                    _ptr(W["wdown"]), _ptr(lm_w), _ptr(emb), _ptr(ph), _ptr(k_cache),
                                    _ptr(v_cache), _ptr(pos), _ptr(u), _ptr(tokens), _ptr(q),
                                    B, r0, d, hq, hkv, I, Lmax, V, K, kp, float(eps), float(theta),
                                    float(temperature), _ptr(ws), ws_len, _stream(stream))
    _raise(st, "sd_semi_ar_draft")
    return tokens, q


def sd_linear_q8(x, wq, scale, bias=None, residual=None, out=None, workspace=None, stream=None):
    """y = x (scale * wq)^T (+ bias) (+ residual): x [R, K] bf16, wq [N, K]
    int8, scale [N] fp32.  Returns y [R, N] fp32."""
    torch = _torch()
    _check(x, "x", dtype=torch.bfloat16, ndim=2)
    _check(wq, "wq", dtype=torch.int8, ndim=2)
    _check(scale, "scale", dtype=torch.float32, ndim=1)
    R, K = x.shape
    N = wq.shape[0]
    if wq.shape[1] != K or scale.shape[0] != N:
        raise ValueError("wq must be [N, K] and scale [N]")
    if bias is not None:
        _check(bias, "bias", dtype=torch.float32, ndim=1)
        if bias.shape[0] != N:
            raise ValueError("bias must be [N]")
    if residual is not None:
        _check(residual, "residual", dtype=torch.float32, ndim=2)
        if tuple(residual.shape) != (R, N):
            raise ValueError("residual must be [R, N]")
    for name, t in (("wq", wq), ("scale", scale), ("bias", bias), ("residual", residual)):
        _same_device(name, t, x.device)
    if out is None:
        out = torch.empty((R, N), dtype=torch.float32, device=x.device)
    _out(out, "out", (R, N), torch.float32, x.device)
    ws_bytes = sd_linear_workspace_size(R, K, N)
    ws, ws_len = _workspace(ws_bytes, x.device, workspace)
    st = library().sd_linear_q8(_ptr(x), _ptr(wq), _ptr(scale), _ptr(bias), _ptr(residual), _ptr(out), R, K, N,
                                _ptr(ws), ws_len, _stream(stream))
    _raise(st, "sd_linear_q8")
    return out


Q8_WEIGHTS = ("fc_w", "wqkv", "wo", "wgu", "wdown")


def sd_semi_ar_layer_q8(u, weights, k_cache, v_cache, pos, hq, hkv, eps, theta, out=None, workspace=None,
                        stream=None):
    """sd_semi_ar_layer of the int8 draft: weights holds int8 fc_w, wqkv, wo,
    wgu, wdown and their fp32 row scales under the names + "_s"."""
    torch = _torch()
    _check(u, "u", dtype=torch.bfloat16, ndim=3)
    B, r, d2 = u.shape
    d = d2 // 2
    for name in Q8_WEIGHTS:
        _check(weights[name], name, dtype=torch.int8, ndim=2)
        _check(weights[name + "_s"], name + "_s", dtype=torch.float32, ndim=1)
        if weights[name + "_s"].shape[0] != weights[name].shape[0]:
            raise ValueError(f"{name}_s must hold one scale per row of {name}")
    for name in ("fc_b", "ln1", "ln2"):
        _check(weights[name], name, dtype=torch.float32, ndim=1)
    _check(k_cache, "k_cache", dtype=torch.bfloat16, ndim=4)
    _check(v_cache, "v_cache", dtype=torch.bfloat16, ndim=4)
    _check(pos, "pos", dtype=torch.int32, ndim=1)
    Lmax = k_cache.shape[1]
    I = weights["wdown"].shape[1]
    D = d // hq
    shapes = {"fc_w": (d, 2 * d), "wqkv": ((hq + 2 * hkv) * D, d), "wo": (d, hq * D), "wgu": (2 * I, d),
              "wdown": (d, I)}
    for name, shp in shapes.items():
        if tuple(weights[name].shape) != shp:
            raise ValueError(f"{name} must be {shp}, got {tuple(weights[name].shape)}")
    for name in ("fc_b", "ln1", "ln2"):
        if tuple(weights[name].shape) != (d,):
            raise ValueError(f"{name} must be ({d},)")
    if tuple(k_cache.shape) != (B, Lmax, hkv, D) or tuple(v_cache.shape) != (B, Lmax, hkv, D):
        raise ValueError("caches must be [B, Lmax, hkv, d / hq]")
    if pos.shape[0] != B:
        raise ValueError("pos must be [B]")
    for name, t in [(n, weights[n]) for n in Q8_WEIGHTS] + [
            (n + "_s", weights[n + "_s"]) for n in Q8_WEIGHTS] + [
            (n, weights[n]) for n in ("fc_b", "ln1", "ln2")] + [
            ("k_cache", k_cache), ("v_cache", v_cache), ("pos", pos)]:
        _same_device(name, t, u.device)
    if out is None:
        out = torch.empty((B, r, d), dtype=torch.float32, device=u.device)
    _out(out, "out", (B, r, d), torch.float32, u.device)
    ws_bytes = sd_semi_ar_layer_workspace_size(B, r, d, hq, hkv, I, Lmax)
    ws, ws_len = _workspace(ws_bytes, u.device, workspace)
    W = weights
    st = library().sd_semi_ar_layer_q8(_ptr(u), _ptr(W["fc_w"]), _ptr(W["fc_w_s"]), _ptr(W["fc_b"]),
                                       _ptr(W["ln1"]), _ptr(W["wqkv"]), _ptr(W["wqkv_s"]), _ptr(W["wo"]),
                                       _ptr(W["wo_s"]), _ptr(W["ln2"]), _ptr(W["wgu"]), _ptr(W["wgu_s"]),
                                       _ptr(W["wdown"]), _ptr(W["wdown_s"]), _ptr(k_cache), _ptr(v_cache),
                                       _ptr(pos), _ptr(out), B, r, d, hq, hkv, I, Lmax, float(eps),
                                       float(theta), _ptr(ws), ws_len, _stream(stream))
    _raise(st, "sd_semi_ar_layer_q8")
    return out


def sd_avg_pool_compress(feats, C, out=None, stream=None):
    """Average pooling of feats [B, N, d] (bf16 or fp32) into C contiguous
    token groups.  Returns out [B, C, d] fp32."""
    torch = _torch()
    _check(feats, "feats", ndim=3)
    B, N, d = feats.shape
    if out is None:
        out = torch.empty((B, C, d), dtype=torch.float32, device=feats.device)
    _out(out, "out", (B, C, d), torch.float32, feats.device)
    st = library().sd_avg_pool_compress(_ptr(feats), _ptr(out), B, N, C, d, _dtype_code(feats), _stream(stream))
    _raise(st, "sd_avg_pool_compress")
    return out


# ---------------------------------------- rotary positions, cache append

def _rows(t, name, dtype=None):
    """A [T, H, D] tensor whose rows are dense; they may lie any stride apart
    (a slice of a fused projection).  Returns its shape and that stride in
    elements."""
    if t.dim() != 3:
        raise ValueError(f"{name} must have 3 dimensions, got {t.dim()}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    shape = T, H, D = t.shape
    sT, sH, sD = t.stride()
    if sD == 1 and sH == D and sT >= H * D:
        return shape, sT
    if (D > 1 and sD != 1) or (H > 1 and sH != D) or (T > 1 and sT < H * D):
        raise ValueError(f"{name} must be [T, H, D] with dense rows (any stride between rows)")
    return shape, (sT if T > 1 else H * D)


def _axes(pos, sections, T):
    """(number of axes, sections as a C array or None); pos [axes, T], [T] or None."""
    axes = None
    if pos is not None:
        ndim = pos.dim()
        if ndim not in (1, 2) or pos.shape[-1] != T:
            raise ValueError(f"pos must be [axes, {T}] or [{T}], got {tuple(pos.shape)}")
        _dense(pos, "pos", _torch().int32, ndim)
        axes = pos.shape[0] if ndim == 2 else 1
    if sections is None:
        return 1 if axes is None else axes, None
    n = len(sections)
    if axes is not None and n != axes:
        raise ValueError(f"sections must name the pairs of each of the {axes} axes of pos, got {n}")
    return n, (_c.c_int32 * n)(*sections)


def sd_rope(x, pos, theta, sections=None, per_axis=False, inverse=False, out=None, stream=None):
    """Rotary positions: x [T, H, D] (fp32 or bf16; rows may lie any stride
    apart), pos [T] or [axes, T] int32, sections the pairs of each axis (None:
    one axis, all D / 2).  per_axis restarts the frequencies in every section.
    inverse turns back, which is also the gradient: dx = sd_rope(dy, ...,
    inverse=True).  out may be x (in place).  Returns out [T, H, D]."""
    _on_current("x pos out", x, pos, out)
    shape, xs = _rows(x, "x")
    T, H, D = shape
    dt = _dtype_code(x)
    if pos is None:
        raise ValueError(f"pos must be [axes, {T}] or [{T}], got None")
    axes, secs = _axes(pos, sections, T)
    if out is None:
        ys = H * D
        out = _empty((T, H, D), (ys, D, 1), x.dtype, x.device, stream)
    else:
        out_shape, ys = _rows(out, "out", x.dtype)
        if out_shape != shape:
            raise ValueError(f"out must have shape {tuple(shape)}, got {tuple(out_shape)}")
    st = library().sd_rope(x.data_ptr(), xs, pos.data_ptr(), out.data_ptr(), ys, T, H, D, axes, secs, theta,
                           SD_ROPE_PER_AXIS if per_axis else SD_ROPE_RUNNING, 1 if inverse else 0, dt,
                           _stream(stream))
    _raise(st, "sd_rope")
    return out


def sd_kv_append(q, k, v, k_cache, v_cache, kv_len, theta, pos=None, sections=None, per_axis=False, row_start=None,
                 page_table=None, num_pages=None, q_out=None, stream=None):
    """New rows into the cache: k, v [T, Hkv, D] (views of a fused projection
    allowed), q [T, Hq, D] or None; caches [B, Lmax, Hkv, D], or page pools
    [P, Hkv, 16, D] with page_table [B, max_pages] int32; kv_len [B] int32, the
    lengths after the append.  row_start [B + 1] int32 names each sequence's
    rows (None: T / B rows each, in order).  Keys and queries are rotated at pos
    [T] or [axes, T] int32 (None: their cache position, which behind a shared
    prefix starts at 0 again: give pos there; theta None: not at all), see
    sd_rope.  fp32 rows may go into a bf16 cache.  The caches are
    written in place.  Returns the rotated queries [T, Hq, D] in the cache's
    dtype (None without q)."""
    int32 = _torch().int32
    _on_current("q k v k_cache v_cache kv_len pos row_start page_table q_out", q, k, v, k_cache, v_cache, kv_len, pos,
                row_start, page_table, q_out)
    src, dtype = k.dtype, k_cache.dtype
    shape, ks = _rows(k, "k")
    v_shape, vs = _rows(v, "v", src)
    T, Hkv, D = shape
    _dense(k_cache, "k_cache", dtype, 4)
    _dense(v_cache, "v_cache", dtype, 4)
    _dense(kv_len, "kv_len", int32, 1)
    B = kv_len.shape[0]
    cache = k_cache.shape
    if v_shape != shape:
        raise ValueError("k and v must have the same shape")
    if cache != v_cache.shape:
        raise ValueError("k_cache and v_cache must have the same shape")
    if page_table is None:
        if cache[0] != B or cache[2] != Hkv or cache[3] != D:
            raise ValueError("contiguous caches must be [B, Lmax, Hkv, D]")
        table, Lmax, max_pages, pages = None, cache[1], 0, 0
    else:
        _dense(page_table, "page_table", int32, 2)
        if cache[1] != Hkv or cache[2] != 16 or cache[3] != D or page_table.shape[0] != B:
            raise ValueError("paged caches must be [P, Hkv, 16, D] with a [B, max_pages] table")
        table, Lmax, max_pages, pages = page_table.data_ptr(), 0, page_table.shape[1], _pages(num_pages, k_cache)
    if row_start is not None:
        _dense(row_start, "row_start", int32, 1)
        if row_start.shape[0] != B + 1:
            raise ValueError("row_start must be [B + 1]")
        row_start = row_start.data_ptr()
    elif T % B != 0:
        raise ValueError("without row_start every sequence has T / B rows")
    Hq = qs = 0
    qp = qop = None
    if q is not None:
        q_shape, qs = _rows(q, "q", src)
        Hq = q_shape[1]
        if q_shape[0] != T or q_shape[2] != D:
            raise ValueError("q must be [T, Hq, D] with the rows of k")
        if q_out is None:
            q_out = _empty((T, Hq, D), (Hq * D, D, 1), dtype, k.device, stream)
        else:
            _out(q_out, "q_out", (T, Hq, D), dtype, k.device)
        qp, qop = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out without q")
    axes, secs, p = 0, None, None
    if theta is not None:
        axes, secs = _axes(pos, sections, T)
        p = _ptr(pos)
    st = library().sd_kv_append(qp, qs, k.data_ptr(), ks, v.data_ptr(), vs, qop, k_cache.data_ptr(),
                                v_cache.data_ptr(), row_start, kv_len.data_ptr(), table, max_pages, pages, Lmax, p, T,
                                B, Hq, Hkv, D, axes, secs, theta or 0.0,
                                SD_ROPE_PER_AXIS if per_axis else SD_ROPE_RUNNING, _dtype_code(k),
                                _dtype_code(k_cache), _stream(stream))
    _raise(st, "sd_kv_append")
    return q_out


# ------------------------------------------- verify with shared prefixes

def sd_verify_shared_workspace_size(B, k, Hq, Hkv, D, G, prefix_capacity, capacity, dtype):
    return library().sd_verify_shared_workspace_size(B, k, Hq, Hkv, D, G, prefix_capacity, capacity, dtype)


def _cache_shape(k, v, rows, table, D, dtype, names, num_pages=None):
    """Checks a contiguous cache [rows, L, Hkv, D] or page pools [P, Hkv, 16,
    D] with their table [rows, pages].  Returns (Hkv, capacity, pages of the
    table, pages of the pool, L, the table's address)."""
    _dense(k, names[0], dtype, 4)
    _dense(v, names[1], dtype, 4)
    shape = k.shape
    if shape != v.shape:
        raise ValueError(f"{names[0]} and {names[1]} must have the same shape")
    if table is None:
        if shape[0] != rows or shape[3] != D:
            raise ValueError(f"contiguous {names[0]} must be [{rows}, L, Hkv, {D}], got {tuple(shape)}")
        return shape[2], shape[1], 0, 0, shape[1], None
    _dense(table, names[2], _torch().int32, 2)
    if shape[2] != 16 or shape[3] != D or table.shape[0] != rows:
        raise ValueError(f"paged {names[0]} must be [P, Hkv, 16, {D}] with {names[2]} [{rows}, pages]")
    pages = table.shape[1]
    return shape[1], 16 * pages, pages, _pages(num_pages, k), 0, table.data_ptr()


def sd_verify_shared(q, k_cache, v_cache, kv_len, prefix_len, k_prefix=None, v_prefix=None, prefix_table=None,
                     group_start=None, page_table=None, num_pages=None, scale=None, out_dtype=None, out=None, lse=True,
                     workspace=None, stream=None):
    """Verification attention of sequences in groups that share a prefix.

    Own keys carry the positions that they were appended with: behind a prefix
    that is pos = prefix length + place in the own cache (text), which
    sd_kv_append takes as its pos.

    q [B, k, Hq, D]; own caches [B, Lmax, Hkv, D], or page pools [P, Hkv, 16,
    D] with page_table [B, max_pages]; kv_len [B] counts own keys, the block
    included.  prefix_len [G]; prefixes k_prefix, v_prefix [G, Lmax, Hkv, D], or
    pages of the same pools (k_prefix None) or of pools of their own with
    prefix_table [G, pages].  group_start [G + 1] int32 names each group's
    sequences (None: B / G each).  scale None: 1 / sqrt(D).  out_dtype float32
    (the default) or, for bf16 inputs, bfloat16.
    Returns (out [B, k, Hq, D], lse [B, k, Hq] fp32 or None)."""
    torch = _torch()
    int32, dtype = torch.int32, q.dtype
    _on_current("q k_cache v_cache kv_len prefix_len k_prefix v_prefix prefix_table group_start page_table", q, k_cache,
                v_cache, kv_len, prefix_len, k_prefix, v_prefix, prefix_table, group_start, page_table)
    _dense(q, "q", dtype, 4)
    _dense(kv_len, "kv_len", int32, 1)
    _dense(prefix_len, "prefix_len", int32, 1)
    shape = B, k, Hq, D = q.shape
    G = prefix_len.shape[0]
    if kv_len.shape[0] != B:
        raise ValueError("kv_len needs one entry per sequence")
    if (k_prefix is None) != (v_prefix is None):
        raise ValueError("k_prefix and v_prefix come together")
    own_pool = k_prefix is None
    if own_pool:
        if page_table is None or prefix_table is None:
            raise ValueError("without k_prefix the prefixes are pages of the caches: both tables are needed")
        k_prefix, v_prefix = k_cache, v_cache
    dt = _dtype_code(q)
    Hkv, cap, max_pages, pages, Lmax, table = _cache_shape(k_cache, v_cache, B, page_table, D, dtype,
                                                           ("k_cache", "v_cache", "page_table"), num_pages)
    Hkv_p, pcap, ppages, ppool, pL, ptable = _cache_shape(k_prefix, v_prefix, G, prefix_table, D, dtype,
                                                          ("k_prefix", "v_prefix", "prefix_table"),
                                                          num_pages if own_pool else None)
    if Hkv_p != Hkv:
        raise ValueError("prefixes and caches must have the same KV heads")
    groups = None
    if group_start is not None:
        _dense(group_start, "group_start", int32, 1)
        if group_start.shape[0] != G + 1:
            raise ValueError("group_start must be [G + 1]")
        groups = group_start.data_ptr()
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out_dtype is None:
        out_dtype = torch.float32 if out is None else out.dtype
    if out_dtype != torch.float32 and out_dtype != torch.bfloat16:
        raise TypeError(f"unsupported out_dtype {out_dtype}: use float32 or bfloat16")
    dev = q.device
    if out is None:
        out = _empty((B, k, Hq, D), (k * Hq * D, Hq * D, D, 1), out_dtype, dev, stream)
    else:
        _out(out, "out", shape, out_dtype, dev)
    lse_t = None
    if lse is True:
        lse_t = _empty((B, k, Hq), (k * Hq, Hq, 1), torch.float32, dev, stream)
    elif lse is not None and lse is not False:
        lse_t = _out(lse, "lse", shape[:3], torch.float32, dev)
    lib = library()
    ws, ws_len = _scratch(lib.sd_verify_shared_workspace_size(B, k, Hq, Hkv, D, G, pcap, cap, dt), dev, workspace,
                          stream)
    st = lib.sd_verify_shared(q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), kv_len.data_ptr(), table,
                              max_pages, pages, Lmax, k_prefix.data_ptr(), v_prefix.data_ptr(), prefix_len.data_ptr(),
                              ptable, ppages, ppool, pL, groups, out.data_ptr(), _ptr(lse_t), B, k, Hq, Hkv, D, G,
                              scale, dt, SD_F32 if out_dtype == torch.float32 else SD_BF16, _ptr(ws), ws_len,
                              _stream(stream))
    _raise(st, "sd_verify_shared")
    return out, lse_t
