"""Binding of the C ABI in include/nuq.h.  Argument marshalling only.

The calls of a training step, an exchange or a variance draw go through _nuq_calls (csrc/nuq_calls.cpp), which takes the plain
case in C++; what it declines, and everything else, goes through the checks and ctypes calls below."""
from __future__ import annotations

import ctypes
import operator
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libnuq.so")

_BUILD = ("run `python -c 'import __graft_entry__ as g; g.build()'` (or `python paper_1908_06077_amd/build.py`) first; "
          "there is no fallback path")

if not os.path.exists(_LIB_PATH):
    raise ImportError("libnuq.so is not built: " + _BUILD)


def _check_built(calls_key: int, library_key: int, calls_torch: str, torch_version: str) -> None:
    """_nuq_calls calls the library by its addresses and reads torch's tensors, so it has to be built for both."""
    if calls_key != library_key:
        raise ImportError("_nuq_calls and libnuq.so are built from different versions of nuq.h: " + _BUILD)
    if calls_torch != torch_version:
        raise ImportError("_nuq_calls is built for torch %s, this is %s: " % (calls_torch, torch_version) + _BUILD)


_lib = ctypes.CDLL(_LIB_PATH)

FLAG_CAPACITY, FLAG_NONFINITE, FLAG_MALFORMED = 1, 2, 4
SYNC_BLOCK = 2048
MAX_BUCKET, MAX_S, MAX_WORKERS = 32768, 14, 32

_u64, _u32, _i32, _vp, _f32 = ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int, ctypes.c_void_p, ctypes.c_float
_f64 = ctypes.c_double

_SIGNATURES = {
    "nuq_num_buckets": (_u64, [_u64, _u32]),
    "nuq_workspace_bytes": (_u64, [_u64, _u32, _u32]),
    "nuq_num_sync": (_u32, [_u32, _u32]),
    "nuq_huffman_num_sync": (_u32, [_u32, _u32]),
    "nuq_max_words": (_u64, [_u64, _u32, _u32]),
    "nuq_encode_workspace_bytes": (_u64, [_u32, _u64, _u32, _u32]),
    "nuq_quantize_encode_batch": (_i32, [_u32, _vp, _vp, _u64, _u32, _u32, _u32, _vp, _vp, _vp, _vp, _vp, _vp, _u64, _vp]),
    "nuq_bucket_norms": (_i32, [_vp, _u64, _u32, _vp, _vp]),
    "nuq_quantize": (_i32, [_vp, _u64, _u32, _u32, _u64, _vp, _vp, _vp]),
    "nuq_encode": (_i32, [_vp, _u64, _u32, _u32, _u32, _vp, _vp, _u64, _vp, _vp, _u64, _vp]),
    "nuq_quantize_encode": (_i32, [_vp, _u64, _u32, _u32, _u64, _u32, _vp, _vp, _vp, _u64, _vp, _vp, _u64, _vp]),
    "nuq_quantize_encode_static": (_i32, [_vp, _u64, _u32, _u32, _u64, _u32, _vp, _vp, _vp, _u64, _vp, _vp]),
    "nuq_decode_accumulate": (_i32, [_u32, _vp, _vp, _vp, _vp, _vp, _u64, _u32, _u32, _u32, _f32, _i32, _vp, _vp]),
    "nuq_bucket_norms_linf": (_i32, [_vp, _u64, _u32, _vp, _vp]),
    "nuq_quantize_table": (_i32, [_vp, _u64, _u32, _u32, _vp, _u64, _vp, _vp, _vp]),
    "nuq_quantize_encode_table_batch": (_i32, [_u32, _vp, _vp, _u64, _u32, _u32, _vp, _u32, _u32, _vp, _vp, _vp, _vp, _vp,
                                               _vp, _u64, _vp]),
    "nuq_decode_accumulate_huffman": (_i32, [_u32, _vp, _vp, _vp, _vp, _vp, _u64, _u32, _u32, _u32, _vp, _f32, _i32, _vp,
                                             _vp]),
    "nuq_decode_accumulate_table": (_i32, [_u32, _vp, _vp, _vp, _vp, _vp, _u64, _u32, _u32, _u32, _vp, _f32, _i32, _vp, _vp]),
    "nuq_fixed_words": (_u64, [_u64, _u32, _u32]),
    "nuq_pack_fixed": (_i32, [_vp, _u64, _u32, _u32, _u32, _vp, _vp]),
    "nuq_quantize_pack_fixed_batch": (_i32, [_u32, _vp, _vp, _u64, _u32, _u32, _u32, _vp, _vp, _vp]),
    "nuq_unpack_accumulate_fixed": (_i32, [_u32, _vp, _vp, _u64, _u32, _u32, _u32, _f32, _i32, _vp, _vp]),
    "nuq_quantize_pack_fixed_table_batch": (_i32, [_u32, _vp, _vp, _u64, _u32, _u32, _vp, _u32, _u32, _vp, _vp, _vp]),
    "nuq_unpack_accumulate_fixed_table": (_i32, [_u32, _vp, _vp, _u64, _u32, _u32, _vp, _u32, _f32, _i32, _vp, _vp]),
    "nuq_level_histogram": (_i32, [_vp, _u64, _vp, _vp]),
    "nuq_huffman_lengths": (_i32, [_vp, _u32, _vp]),
    "nuq_huffman_max_words": (_u64, [_u64, _u32]),
    "nuq_encode_huffman_workspace_bytes": (_u64, [_u64, _u32]),
    "nuq_encode_huffman": (_i32, [_vp, _u64, _u32, _u32, _u32, _vp, _vp, _vp, _u64, _vp, _vp, _u64, _vp]),
    "nuq_decode_huffman": (_i32, [_vp, _vp, _vp, _u64, _u32, _u32, _u32, _vp, _vp, _vp]),
    "nuq_encode_huffman_batch_workspace_bytes": (_u64, [_u32, _u64, _u32, _u32]),
    "nuq_quantize_encode_huffman_batch": (_i32, [_u32, _vp, _vp, _u64, _u32, _u32, _u32, _vp, _vp, _vp, _vp, _vp, _vp,
                                                 _vp, _u64, _vp]),
    "nuq_decode_huffman_batch": (_i32, [_u32, _vp, _vp, _vp, _u64, _u32, _u32, _u32, _vp, _vp, _vp]),
    "nuq_average_levels": (_i32, [_u32, _vp, _vp, _u64, _u32, _u32, _f32, _i32, _vp, _vp]),
    "nuq_momentum_step": (_i32, [_vp, _vp, _vp, _u64, _f32, _f32, _f32, _vp]),
    "nuq_decode_momentum_step": (_i32, [_u32, _vp, _vp, _vp, _vp, _vp, _u64, _u32, _u32, _u32, _f32, _f32, _f32, _f32, _vp,
                                        _vp, _vp]),
    "nuq_moments_accumulate": (_i32, [_vp, _vp, _vp, _u64, _vp]),
    "nuq_normalized_variance": (_i32, [_vp, _vp, _u64, _u64, _vp, _u64, _vp, _vp]),
    "nuq_gradient_norm": (_i32, [_u32, _vp, _vp, _u32, _f32, _vp, _u64, _vp, _vp]),
    "nuq_adamw_step": (_i32, [_u32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _u32, _u32, _f64, _f64, _f64, _f64, _u64, _vp, _vp]),
    "nuq_state_blocks": (_u64, [_u64]),
    "nuq_adamw_step_coded": (_i32, [_u32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _u32, _u32, _f64, _f64, _f64, _f64, _u64, _vp,
                                    _vp]),
    "nuq_adamw_state_values": (_i32, [_vp, _vp, _vp, _u64, _vp, _vp, _vp]),
    "nuq_layer_norm_forward": (_i32, [_vp, _u64, _vp, _u64, _vp, _vp, _u64, _u32, _f32, _u32, _u32, _vp, _u64, _vp, _u64, _vp,
                                      _vp, _vp]),
    "nuq_layer_norm_workspace_bytes": (_u64, [_u64, _u32]),
    "nuq_layer_norm_backward": (_i32, [_vp, _u64, _vp, _u64, _vp, _vp, _vp, _vp, _u64, _u64, _u32, _u32, _u32, _vp, _u64, _vp,
                                       _vp, _vp, _u64, _vp]),
    "nuq_dropout": (_i32, [_vp, _u64, _vp, _u64, _u64, _u32, _u32, _f64, _u64, _vp, _vp, _u64, _vp]),
    "nuq_residual_norm_forward": (_i32, [_vp, _u64, _vp, _u64, _u32, _vp, _vp, _vp, _u32, _vp, _vp, _u64, _u32, _f32, _f32, _f32,
                                         _f64, _u64, _vp, _u32, _u32, _vp, _u64, _vp, _u64, _vp, _vp]),
    "nuq_residual_norm_workspace_bytes": (_u64, [_u64, _u32]),
    "nuq_residual_norm_backward": (_i32, [_vp, _u64, _vp, _u64, _vp, _u64, _vp, _u64, _u32, _vp, _vp, _vp, _u32, _vp, _u64, _u32,
                                          _f32, _f32, _f64, _u64, _vp, _u32, _u32, _vp, _vp, _u64, _vp, _u64, _vp, _vp, _vp, _vp,
                                          _vp, _vp, _u64, _vp]),
    "nuq_linear_cross_entropy_workspace_bytes": (_u64, [_vp, _u64, _vp, _u64, _u64, _u32, _u32, _u32, _i32]),
    "nuq_linear_cross_entropy_forward": (_i32, [_vp, _u64, _vp, _u64, _u64, _u32, _u32, _u32, _vp, ctypes.c_int64, _f32, _vp, _vp, _vp,
                                                _vp, _u64, _vp]),
    "nuq_linear_cross_entropy_backward": (_i32, [_vp, _u64, _vp, _u64, _u64, _u32, _u32, _u32, _vp, ctypes.c_int64, _f32, _vp, _vp, _i32,
                                                 _vp, _vp, _u64, _vp, _u64, _vp, _u64, _vp]),
    "nuq_last_error_flags": (_i32, [_vp, _vp]),
    "nuq_encode_shape": (_i32, [_u32, _u32, _u64, _u32, _u32, _u32, _vp, _u32, _vp]),
    "nuq_decode_tile": (_u32, [_u32, _u64, _u32, _u32, _u32, _i32, _u32]),
    "nuq_timing_begin": (_i32, [_u32]),
    "nuq_timing_collect": (_i32, [_vp, _vp, _u32, _vp]),
}
for _name, (_res, _args) in _SIGNATURES.items():
    _fn = getattr(_lib, _name)
    _fn.restype = _res
    _fn.argtypes = _args


try:
    from . import _nuq_calls as _calls  # noqa: E402
except ImportError as e:
    raise ImportError("_nuq_calls is not built for this Python and torch (%s): " % e + _BUILD) from e
_check_built(_calls.header_key, ctypes.c_uint64.in_dll(_lib, "nuq_header_key").value, _calls.torch_version,
             torch.__version__)

_calls.bind(tuple(ctypes.cast(getattr(_lib, n), ctypes.c_void_p).value for n in _calls.names()),
            torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)


def library_path() -> str:
    return _LIB_PATH


def exported_symbols() -> list[str]:
    return sorted(_SIGNATURES)


class NuqError(RuntimeError):
    def __init__(self, fn: str, code: int):
        names = {-1: "NUQ_EINVAL", -2: "NUQ_ECAPACITY", -3: "NUQ_ENONFINITE", -4: "NUQ_EHIP"}
        super().__init__("%s returned %s" % (fn, names.get(code, str(code))))
        self.code = code


def _check(fn: str, code: int) -> None:
    if code != 0:
        raise NuqError(fn, code)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


_on_device = operator.attrgetter("is_cuda")


def _ptr(t: torch.Tensor | None, dtype: torch.dtype | None = None, need: int = 0, what: str = "tensor") -> int:
    """Device address of t after checking what the kernels take on trust: placement, contiguity, element type and
    that it holds at least `need` elements."""
    if t is None:
        if need:
            raise ValueError("%s is needed (%d elements)" % (what, need))
        return 0
    if dtype is not None and t.dtype is not dtype:
        raise ValueError("%s: expected dtype %s, got %s" % (what, dtype, t.dtype))
    if need and t.numel() < need:
        raise ValueError("%s holds %d elements, %d are needed" % (what, t.numel(), need))
    if not _on_device(t) or not t.is_contiguous():
        raise ValueError("%s: expected a contiguous device tensor" % what)
    return t.data_ptr()


def _sizes(d: int, bucket: int, sync_stride: int, huffman: bool = False) -> tuple[int, int]:
    """(buckets, sync entries of a whole message) for the size checks; (0, 0) for arguments the library rejects."""
    B = _lib.nuq_num_buckets(d, bucket)
    per = (_lib.nuq_huffman_num_sync if huffman else _lib.nuq_num_sync)(bucket, sync_stride) if bucket else 0
    return B, B * per


def _message_arrays(messages, d: int, bucket: int, sync_stride: int, huffman: bool = False, norms: bool = True):
    """ctypes pointer arrays (norms, bit_off, words, words_len, sync) of K messages, every tensor checked against the
    size that d, bucket and sync_stride imply."""
    K = len(messages)
    B, nsync = _sizes(d, bucket, sync_stride, huffman)
    addresses = ctypes.c_uint64 * K                      # (one array type: addresses and lengths alike)
    ptr, f32, i32, i64 = _ptr, torch.float32, torch.int32, torch.int64
    nrm, off, wrd, num, syn = [], [], [], [], []
    for m in messages:
        words = m.words
        if norms:
            nrm.append(ptr(m.norms, f32, B, "norms"))
        off.append(ptr(m.bit_off, i64, B + 1, "bit_off"))
        wrd.append(ptr(words, i32, 0, "words"))
        num.append(words.numel())
        syn.append(ptr(m.sync, i32, nsync, "sync"))
    return (addresses(*nrm) if norms else None, addresses(*off), addresses(*wrd), addresses(*num), addresses(*syn))


# ------------------------------------------------------------------ sizes (host only)

def nuq_num_buckets(d: int, bucket: int) -> int:
    return _lib.nuq_num_buckets(d, bucket)


def nuq_num_sync(bucket: int, sync_stride: int) -> int:
    return _lib.nuq_num_sync(bucket, sync_stride)


def nuq_huffman_num_sync(bucket: int, sync_stride: int) -> int:
    return _lib.nuq_huffman_num_sync(bucket, sync_stride)


def nuq_max_words(d: int, bucket: int, s: int) -> int:
    return _lib.nuq_max_words(d, bucket, s)


def nuq_encode_workspace_bytes(K: int, d: int, bucket: int, s: int) -> int:
    return _lib.nuq_encode_workspace_bytes(K, d, bucket, s)


def nuq_workspace_bytes(d: int, bucket: int, K: int) -> int:
    return _lib.nuq_workspace_bytes(d, bucket, K)


# ------------------------------------------------------------------------- the path

def nuq_bucket_norms(v: torch.Tensor, bucket: int, norms: torch.Tensor) -> None:
    _check("nuq_bucket_norms",
           _lib.nuq_bucket_norms(_ptr(v, torch.float32), v.numel(), bucket,
                                 _ptr(norms, torch.float32, nuq_num_buckets(v.numel(), bucket), "norms"), _stream()))


def nuq_quantize(v: torch.Tensor, bucket: int, s: int, seed: int, norms: torch.Tensor, q: torch.Tensor) -> None:
    _check("nuq_quantize",
           _lib.nuq_quantize(_ptr(v, torch.float32), v.numel(), bucket, s, seed & (2 ** 64 - 1),
                             _ptr(norms, torch.float32, nuq_num_buckets(v.numel(), bucket), "norms"),
                             _ptr(q, torch.uint8, v.numel(), "q"), _stream()))


@dataclass
class Message:
    """One worker's encoded gradient: device tensors laid out as include/nuq.h describes."""
    norms: torch.Tensor       # float32 [B]
    bit_off: torch.Tensor     # int64 [B+1] (u64 bit pattern)
    words: torch.Tensor       # int32 [words_cap] (u32 bit pattern)
    sync: torch.Tensor | None  # int32 [B*nsync]


def nuq_encode(q: torch.Tensor, bucket: int, s: int, sync_stride: int, bit_off: torch.Tensor, words: torch.Tensor,
               sync: torch.Tensor | None, workspace: torch.Tensor) -> None:
    B, nsync = _sizes(q.numel(), bucket, sync_stride)
    _check("nuq_encode",
           _lib.nuq_encode(_ptr(q, torch.uint8), q.numel(), bucket, s, sync_stride,
                           _ptr(bit_off, torch.int64, B + 1, "bit_off"), _ptr(words, torch.int32), words.numel(),
                           _ptr(sync, torch.int32, nsync, "sync"), _ptr(workspace),
                           workspace.numel() * workspace.element_size(), _stream()))


def nuq_quantize_encode(v: torch.Tensor, bucket: int, s: int, seed: int, sync_stride: int, norms: torch.Tensor,
                        bit_off: torch.Tensor, words: torch.Tensor, sync: torch.Tensor | None,
                        workspace: torch.Tensor) -> None:
    B, nsync = _sizes(v.numel(), bucket, sync_stride)
    _check("nuq_quantize_encode",
           _lib.nuq_quantize_encode(_ptr(v, torch.float32), v.numel(), bucket, s, seed & (2 ** 64 - 1), sync_stride,
                                    _ptr(norms, torch.float32, B, "norms"), _ptr(bit_off, torch.int64, B + 1, "bit_off"),
                                    _ptr(words, torch.int32), words.numel(), _ptr(sync, torch.int32, nsync, "sync"),
                                    _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()))


STATIC_WORKSPACE_BYTES = 32 << 20


def nuq_quantize_encode_static(v: torch.Tensor, bucket: int, s: int, seed: int, sync_stride: int, norms: torch.Tensor,
                               bit_off: torch.Tensor, words: torch.Tensor, sync: torch.Tensor | None) -> None:
    """nuq_quantize_encode with the library's own workspace: the call allocates nothing."""
    B, nsync = _sizes(v.numel(), bucket, sync_stride)
    _check("nuq_quantize_encode_static",
           _lib.nuq_quantize_encode_static(_ptr(v, torch.float32), v.numel(), bucket, s, seed & (2 ** 64 - 1),
                                           sync_stride, _ptr(norms, torch.float32, B, "norms"),
                                           _ptr(bit_off, torch.int64, B + 1, "bit_off"), _ptr(words, torch.int32),
                                           words.numel(), _ptr(sync, torch.int32, nsync, "sync"), _stream()))


def nuq_quantize_encode_batch(vs: list[torch.Tensor], bucket: int, s: int, seeds: list[int], sync_stride: int,
                              messages: list["Message"], workspace: torch.Tensor) -> None:
    code = _calls.quantize_encode_batch(vs, bucket, s, seeds, sync_stride, messages, workspace)
    if code is not None:
        return _check("nuq_quantize_encode_batch", code)
    K = len(vs)
    d = vs[0].numel()
    if any([v.numel() != d for v in vs]) or len(seeds) != K or len(messages) != K:
        raise ValueError("K gradients of equal length, K seeds and K messages are needed")
    u64 = ctypes.c_uint64 * K
    norms, offs, words, caps, sync = _message_arrays(messages, d, bucket, sync_stride)
    _check("nuq_quantize_encode_batch",
           _lib.nuq_quantize_encode_batch(K, u64(*[_ptr(v, torch.float32) for v in vs]),
                                          u64(*[x & (2 ** 64 - 1) for x in seeds]), d, bucket, s, sync_stride,
                                          norms, offs, words, caps, sync, _ptr(workspace),
                                          workspace.numel() * workspace.element_size(), _stream()))


def nuq_decode_accumulate(messages: list[Message], d: int, bucket: int, s: int, sync_stride: int, scale: float,
                          accumulate: bool, out: torch.Tensor) -> None:
    code = _calls.decode_accumulate(messages, d, bucket, s, sync_stride, scale, accumulate, out)
    if code is not None:
        return _check("nuq_decode_accumulate", code)
    K = len(messages)
    norms, offs, words, lens, sync = _message_arrays(messages, d, bucket, sync_stride)
    if out.numel() != d:
        raise ValueError("out must hold d floats")
    _check("nuq_decode_accumulate",
           _lib.nuq_decode_accumulate(K, norms, offs, words, lens, sync, d, bucket, s, sync_stride, float(scale),
                                      1 if accumulate else 0, _ptr(out, torch.float32), _stream()))


# ------------------------------------------- other level sequences, maximum norm

def _levels(levels, s: int):
    if len(levels) != s + 2:
        raise ValueError("a level table holds s + 2 values")
    return (ctypes.c_float * (s + 2))(*[float(x) for x in levels])


def nuq_bucket_norms_linf(v: torch.Tensor, bucket: int, norms: torch.Tensor) -> None:
    _check("nuq_bucket_norms_linf",
           _lib.nuq_bucket_norms_linf(_ptr(v, torch.float32), v.numel(), bucket,
                                      _ptr(norms, torch.float32, nuq_num_buckets(v.numel(), bucket), "norms"),
                                      _stream()))


def nuq_quantize_table(v: torch.Tensor, bucket: int, levels, seed: int, norms: torch.Tensor, q: torch.Tensor) -> None:
    s = len(levels) - 2
    _check("nuq_quantize_table",
           _lib.nuq_quantize_table(_ptr(v, torch.float32), v.numel(), bucket, s, _levels(levels, s),
                                   seed & (2 ** 64 - 1),
                                   _ptr(norms, torch.float32, nuq_num_buckets(v.numel(), bucket), "norms"),
                                   _ptr(q, torch.uint8, v.numel(), "q"), _stream()))


NORM_L2, NORM_LINF = 0, 1


def nuq_quantize_encode_table_batch(vs: list[torch.Tensor], bucket: int, levels, norm_kind: int, seeds: list[int],
                                    sync_stride: int, messages: list["Message"], workspace: torch.Tensor) -> None:
    code = _calls.quantize_encode_table_batch(vs, bucket, levels, norm_kind, seeds, sync_stride, messages, workspace)
    if code is not None:
        return _check("nuq_quantize_encode_table_batch", code)
    K = len(vs)
    d = vs[0].numel()
    s = len(levels) - 2
    if any(v.numel() != d for v in vs) or len(seeds) != K or len(messages) != K:
        raise ValueError("K gradients of equal length, K seeds and K messages are needed")
    arr = lambda ts, dt=None: (ctypes.c_void_p * K)(*[_ptr(t, dt) for t in ts])
    u64s = lambda xs: (ctypes.c_uint64 * K)(*[x & (2 ** 64 - 1) for x in xs])
    norms, offs, words, caps, sync = _message_arrays(messages, d, bucket, sync_stride)
    _check("nuq_quantize_encode_table_batch",
           _lib.nuq_quantize_encode_table_batch(K, arr(vs, torch.float32), u64s(seeds), d, bucket, s,
                                                _levels(levels, s), norm_kind, sync_stride, norms, offs, words, caps,
                                                sync, _ptr(workspace), workspace.numel() * workspace.element_size(),
                                                _stream()))


def nuq_decode_accumulate_table(messages: list[Message], d: int, bucket: int, levels, sync_stride: int, scale: float,
                                accumulate: bool, out: torch.Tensor) -> None:
    code = _calls.decode_accumulate_table(messages, d, bucket, levels, sync_stride, scale, accumulate, out)
    if code is not None:
        return _check("nuq_decode_accumulate_table", code)
    K = len(messages)
    s = len(levels) - 2
    norms, offs, words, lens, sync = _message_arrays(messages, d, bucket, sync_stride)
    if out.numel() != d:
        raise ValueError("out must hold d floats")
    _check("nuq_decode_accumulate_table",
           _lib.nuq_decode_accumulate_table(K, norms, offs, words, lens, sync, d, bucket, s, sync_stride,
                                            _levels(levels, s), float(scale), 1 if accumulate else 0,
                                            _ptr(out, torch.float32), _stream()))


# --------------------------------------------------------- fixed-width coding

def nuq_fixed_words(d: int, bucket: int, b: int) -> int:
    return _lib.nuq_fixed_words(d, bucket, b)


def nuq_pack_fixed(q: torch.Tensor, bucket: int, s: int, b: int, packed: torch.Tensor) -> None:
    _check("nuq_pack_fixed",
           _lib.nuq_pack_fixed(_ptr(q, torch.uint8), q.numel(), bucket, s, b, _ptr(packed, torch.int32), _stream()))


def nuq_quantize_pack_fixed_batch(vs: list[torch.Tensor], bucket: int, s: int, b: int, seeds: list[int],
                                  norms: list[torch.Tensor], packed: list[torch.Tensor]) -> None:
    code = _calls.quantize_pack_fixed_batch(vs, bucket, s, b, seeds, norms, packed)
    if code is not None:
        return _check("nuq_quantize_pack_fixed_batch", code)
    K = len(vs)
    d = vs[0].numel()
    if any(v.numel() != d for v in vs) or len(seeds) != K or len(norms) != K or len(packed) != K:
        raise ValueError("K gradients of equal length, K seeds, K norm arrays and K packed arrays are needed")
    arr = lambda ts, dt: (ctypes.c_void_p * K)(*[_ptr(t, dt) for t in ts])
    _check("nuq_quantize_pack_fixed_batch",
           _lib.nuq_quantize_pack_fixed_batch(K, arr(vs, torch.float32),
                                              (ctypes.c_uint64 * K)(*[x & (2 ** 64 - 1) for x in seeds]), d, bucket,
                                              s, b, arr(norms, torch.float32), arr(packed, torch.int32), _stream()))


def nuq_unpack_accumulate_fixed(norms: list[torch.Tensor], packed: list[torch.Tensor], d: int, bucket: int, s: int,
                                b: int, scale: float, accumulate: bool, out: torch.Tensor) -> None:
    code = _calls.unpack_accumulate_fixed(norms, packed, d, bucket, s, b, scale, accumulate, out)
    if code is not None:
        return _check("nuq_unpack_accumulate_fixed", code)
    K = len(norms)
    arr = lambda ts, dt: (ctypes.c_void_p * K)(*[_ptr(t, dt) for t in ts])
    if out.numel() != d:
        raise ValueError("out must hold d floats")
    _check("nuq_unpack_accumulate_fixed",
           _lib.nuq_unpack_accumulate_fixed(K, arr(norms, torch.float32), arr(packed, torch.int32), d, bucket, s, b,
                                            float(scale), 1 if accumulate else 0, _ptr(out, torch.float32), _stream()))


def nuq_quantize_pack_fixed_table_batch(vs: list[torch.Tensor], bucket: int, levels, norm_kind: int, b: int,
                                        seeds: list[int], norms: list[torch.Tensor], packed: list[torch.Tensor]) -> None:
    code = _calls.quantize_pack_fixed_table_batch(vs, bucket, levels, norm_kind, b, seeds, norms, packed)
    if code is not None:
        return _check("nuq_quantize_pack_fixed_table_batch", code)
    K = len(vs)
    d = vs[0].numel()
    s = len(levels) - 2
    if any(v.numel() != d for v in vs) or len(seeds) != K or len(norms) != K or len(packed) != K:
        raise ValueError("K gradients of equal length, K seeds, K norm arrays and K packed arrays are needed")
    B, words = nuq_num_buckets(d, bucket), nuq_fixed_words(d, bucket, b)
    _check("nuq_quantize_pack_fixed_table_batch",
           _lib.nuq_quantize_pack_fixed_table_batch(
               K, (ctypes.c_void_p * K)(*[_ptr(v, torch.float32) for v in vs]),
               (ctypes.c_uint64 * K)(*[x & (2 ** 64 - 1) for x in seeds]), d, bucket, s, _levels(levels, s), norm_kind, b,
               (ctypes.c_void_p * K)(*[_ptr(t, torch.float32, B, "norms") for t in norms]),
               (ctypes.c_void_p * K)(*[_ptr(t, torch.int32, words, "packed") for t in packed]), _stream()))


def nuq_unpack_accumulate_fixed_table(norms: list[torch.Tensor], packed: list[torch.Tensor], d: int, bucket: int,
                                      levels, b: int, scale: float, accumulate: bool, out: torch.Tensor) -> None:
    code = _calls.unpack_accumulate_fixed_table(norms, packed, d, bucket, levels, b, scale, accumulate, out)
    if code is not None:
        return _check("nuq_unpack_accumulate_fixed_table", code)
    K = len(norms)
    s = len(levels) - 2
    if out.numel() != d or len(packed) != K:
        raise ValueError("K norm arrays, K packed arrays and d floats of output are needed")
    B, words = nuq_num_buckets(d, bucket), nuq_fixed_words(d, bucket, b)
    _check("nuq_unpack_accumulate_fixed_table",
           _lib.nuq_unpack_accumulate_fixed_table(
               K, (ctypes.c_void_p * K)(*[_ptr(t, torch.float32, B, "norms") for t in norms]),
               (ctypes.c_void_p * K)(*[_ptr(t, torch.int32, words, "packed") for t in packed]), d, bucket, s,
               _levels(levels, s), b, float(scale), 1 if accumulate else 0, _ptr(out, torch.float32), _stream()))


# -------------------------------------------------------- Huffman-coded levels

def nuq_level_histogram(q: torch.Tensor, hist: torch.Tensor) -> None:
    """hist: int64[16] on the device, overwritten."""
    if hist.numel() < 16:
        raise ValueError("hist holds 16 counters")
    _check("nuq_level_histogram",
           _lib.nuq_level_histogram(_ptr(q, torch.uint8), q.numel(), _ptr(hist, torch.int64), _stream()))


def nuq_huffman_lengths(hist: list[int], s: int) -> list[int]:
    """Host arithmetic: code lengths of the level indices 0..s+1 from their counts."""
    if len(hist) != s + 2:
        raise ValueError("one count per level index 0..s+1")
    h = (ctypes.c_uint64 * (s + 2))(*[int(x) for x in hist])
    out = (ctypes.c_uint8 * (s + 2))()
    _check("nuq_huffman_lengths", _lib.nuq_huffman_lengths(h, s, out))
    return list(out)


def nuq_huffman_max_words(d: int, bucket: int) -> int:
    return _lib.nuq_huffman_max_words(d, bucket)


def nuq_encode_huffman_workspace_bytes(d: int, bucket: int) -> int:
    return _lib.nuq_encode_huffman_workspace_bytes(d, bucket)


def _lengths(lengths, s: int):
    if len(lengths) != s + 2:
        raise ValueError("one code length per level index 0..s+1")
    return (ctypes.c_uint8 * (s + 2))(*[int(x) for x in lengths])


def nuq_encode_huffman(q: torch.Tensor, bucket: int, s: int, sync_stride: int, lengths, bit_off: torch.Tensor,
                       words: torch.Tensor, sync: torch.Tensor | None, workspace: torch.Tensor) -> None:
    _check("nuq_encode_huffman",
           _lib.nuq_encode_huffman(_ptr(q, torch.uint8), q.numel(), bucket, s, sync_stride, _lengths(lengths, s),
                                   _ptr(bit_off, torch.int64), _ptr(words, torch.int32), words.numel(), _ptr(sync),
                                   _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()))


def nuq_decode_huffman(bit_off: torch.Tensor, words: torch.Tensor, sync: torch.Tensor | None, d: int, bucket: int,
                       s: int, sync_stride: int, lengths, q: torch.Tensor) -> None:
    if q.numel() != d:
        raise ValueError("q must hold d bytes")
    _check("nuq_decode_huffman",
           _lib.nuq_decode_huffman(_ptr(bit_off, torch.int64), _ptr(words, torch.int32), _ptr(sync), d, bucket, s,
                                   sync_stride, _lengths(lengths, s), _ptr(q, torch.uint8), _stream()))


def nuq_encode_huffman_batch_workspace_bytes(K: int, d: int, bucket: int, s: int) -> int:
    return _lib.nuq_encode_huffman_batch_workspace_bytes(K, d, bucket, s)


def nuq_quantize_encode_huffman_batch(vs: list[torch.Tensor], bucket: int, s: int, seeds: list[int], sync_stride: int,
                                      lengths, messages: list["Message"], workspace: torch.Tensor) -> None:
    code = _calls.quantize_encode_huffman_batch(vs, bucket, s, seeds, sync_stride, lengths, messages, workspace)
    if code is not None:
        return _check("nuq_quantize_encode_huffman_batch", code)
    K = len(vs)
    d = vs[0].numel()
    if any(v.numel() != d for v in vs) or len(seeds) != K or len(messages) != K:
        raise ValueError("K gradients of equal length, K seeds and K messages are needed")
    arr = lambda ts, dt=None: (ctypes.c_void_p * K)(*[_ptr(t, dt) for t in ts])
    u64s = lambda xs: (ctypes.c_uint64 * K)(*[x & (2 ** 64 - 1) for x in xs])
    _check("nuq_quantize_encode_huffman_batch",
           _lib.nuq_quantize_encode_huffman_batch(K, arr(vs, torch.float32), u64s(seeds), d, bucket, s, sync_stride,
                                                  _lengths(lengths, s),
                                                  arr([m.norms for m in messages], torch.float32),
                                                  arr([m.bit_off for m in messages], torch.int64),
                                                  arr([m.words for m in messages], torch.int32),
                                                  u64s([m.words.numel() for m in messages]),
                                                  arr([m.sync for m in messages]), _ptr(workspace),
                                                  workspace.numel() * workspace.element_size(), _stream()))


def nuq_decode_huffman_batch(messages: list[Message], d: int, bucket: int, s: int, sync_stride: int, lengths,
                             qs: list[torch.Tensor]) -> None:
    K = len(messages)
    if len(qs) != K or any(q.numel() != d for q in qs):
        raise ValueError("K messages and K byte arrays of d entries are needed")
    arr = lambda ts, dt=None: (ctypes.c_void_p * K)(*[_ptr(t, dt) for t in ts])
    _check("nuq_decode_huffman_batch",
           _lib.nuq_decode_huffman_batch(K, arr([m.bit_off for m in messages], torch.int64),
                                         arr([m.words for m in messages], torch.int32),
                                         arr([m.sync for m in messages]), d, bucket, s, sync_stride,
                                         _lengths(lengths, s), arr(qs, torch.uint8), _stream()))


def nuq_decode_accumulate_huffman(messages: list[Message], d: int, bucket: int, s: int, sync_stride: int, lengths,
                                  scale: float, accumulate: bool, out: torch.Tensor) -> None:
    code = _calls.decode_accumulate_huffman(messages, d, bucket, s, sync_stride, lengths, scale, accumulate, out)
    if code is not None:
        return _check("nuq_decode_accumulate_huffman", code)
    K = len(messages)
    norms, offs, words, lens, sync = _message_arrays(messages, d, bucket, sync_stride, huffman=True)
    if out.numel() != d:
        raise ValueError("out must hold d floats")
    _check("nuq_decode_accumulate_huffman",
           _lib.nuq_decode_accumulate_huffman(K, norms, offs, words, lens, sync, d, bucket, s, sync_stride,
                                              _lengths(lengths, s), float(scale), 1 if accumulate else 0,
                                              _ptr(out, torch.float32), _stream()))


def nuq_average_levels(norms: list[torch.Tensor], qs: list[torch.Tensor], d: int, bucket: int, s: int, scale: float,
                       accumulate: bool, out: torch.Tensor) -> None:
    K = len(norms)
    arr = lambda ts, dt: (ctypes.c_void_p * K)(*[_ptr(t, dt) for t in ts])
    if out.numel() != d or len(qs) != K:
        raise ValueError("K norm arrays, K byte arrays and d floats of output are needed")
    _check("nuq_average_levels",
           _lib.nuq_average_levels(K, arr(norms, torch.float32), arr(qs, torch.uint8), d, bucket, s, float(scale),
                                   1 if accumulate else 0, _ptr(out, torch.float32), _stream()))


# --------------------------------- parameter update and variance diagnostic

VARIANCE_WORKSPACE_BYTES = 16384


def nuq_momentum_step(w: torch.Tensor, yl: torch.Tensor, g: torch.Tensor, alpha: float, mu: float, l: float) -> None:
    d = w.numel()
    if yl.numel() != d or g.numel() != d:
        raise ValueError("w, yl and g hold d floats each")
    _check("nuq_momentum_step",
           _lib.nuq_momentum_step(_ptr(w, torch.float32), _ptr(yl, torch.float32), _ptr(g, torch.float32), d,
                                  float(alpha), float(mu), float(l), _stream()))


def nuq_decode_momentum_step(messages: list[Message], d: int, bucket: int, s: int, sync_stride: int, scale: float,
                             alpha: float, mu: float, l: float, w: torch.Tensor, yl: torch.Tensor) -> None:
    code = _calls.decode_momentum_step(messages, d, bucket, s, sync_stride, scale, alpha, mu, l, w, yl)
    if code is not None:
        return _check("nuq_decode_momentum_step", code)
    K = len(messages)
    norms, offs, words, lens, sync = _message_arrays(messages, d, bucket, sync_stride)
    if w.numel() != d or yl.numel() != d:
        raise ValueError("w and yl hold d floats each")
    _check("nuq_decode_momentum_step",
           _lib.nuq_decode_momentum_step(K, norms, offs, words, lens, sync, d, bucket,
                                         s, sync_stride, float(scale), float(alpha), float(mu), float(l),
                                         _ptr(w, torch.float32), _ptr(yl, torch.float32), _stream()))


def nuq_moments_accumulate(g: torch.Tensor, total: torch.Tensor, total_sq: torch.Tensor) -> None:
    code = _calls.moments_accumulate(g, total, total_sq)
    if code is not None:
        return _check("nuq_moments_accumulate", code)
    d = g.numel()
    if total.numel() != d or total_sq.numel() != d:
        raise ValueError("the moment sums hold d doubles each")
    _check("nuq_moments_accumulate",
           _lib.nuq_moments_accumulate(_ptr(g, torch.float32), _ptr(total, torch.float64),
                                       _ptr(total_sq, torch.float64), d, _stream()))


def nuq_normalized_variance(total: torch.Tensor, total_sq: torch.Tensor, M: int, workspace: torch.Tensor,
                            out2: torch.Tensor) -> None:
    d = total.numel()
    if total_sq.numel() != d or out2.numel() != 2:
        raise ValueError("two moment sums of d doubles and two doubles of output are needed")
    _check("nuq_normalized_variance",
           _lib.nuq_normalized_variance(_ptr(total, torch.float64), _ptr(total_sq, torch.float64), d, M,
                                        _ptr(workspace), workspace.numel() * workspace.element_size(),
                                        _ptr(out2, torch.float64), _stream()))


# ------------------------------------------ AdamW, the gradients' norm, layer norm

GRADIENT_NORM_WORKSPACE_BYTES = 65536
STATE_BLOCK = 256

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _type(t: torch.Tensor, what: str) -> int:
    try:
        return _TYPES[t.dtype]
    except KeyError:
        raise ValueError("%s: expected float32, bfloat16 or float16, got %s" % (what, t.dtype)) from None


def _tensors(ts, what: str, like: list[int] | None = None, dtype: torch.dtype | None = None):
    """(pointer array, element counts) of device tensors of one type, each as long as `like` says."""
    ts = list(ts)
    if like is not None and len(ts) != len(like):
        raise ValueError("%s: %d tensors, %d are needed" % (what, len(ts), len(like)))
    counts = [t.numel() for t in ts]
    dtype = dtype or (ts[0].dtype if ts else None)
    for i, t in enumerate(ts):
        if like is not None and counts[i] != like[i]:
            raise ValueError("%s[%d] holds %d elements, %d are needed" % (what, i, counts[i], like[i]))
    return (ctypes.c_void_p * len(ts))(*[_ptr(t, dtype, 0, what) for t in ts]), counts


def nuq_gradient_norm(grads, max_norm: float, workspace: torch.Tensor, out: torch.Tensor) -> None:
    """out[0] <- the norm of all `grads` taken as one vector, out[1] <- min(1, max_norm / norm), both on the device."""
    code = _calls.gradient_norm(grads, max_norm, workspace, out)
    if code is not None:
        return _check("nuq_gradient_norm", code)
    pointers, counts = _tensors(grads, "grads")
    _check("nuq_gradient_norm",
           _lib.nuq_gradient_norm(len(counts), pointers, (_u64 * len(counts))(*counts), _type(grads[0], "grads") if counts else 0,
                                  float(max_norm), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                  _ptr(out, torch.float32, 2, "out"), _stream()))


def _step_arguments(ws, grads, decays, coefficient, copies):
    w, counts = _tensors(ws, "ws", dtype=torch.float32)
    g, _ = _tensors(grads, "grads", counts)
    T = len(counts)
    if decays is not None and len(decays) != T:
        raise ValueError("one weight decay per tensor")
    copy, copy_type = None, 0
    if copies is not None:
        copy, _ = _tensors(copies, "copies", counts)
        copy_type = _type(copies[0], "copies") if T else 1
    return (w, g, counts, copy, (_u64 * T)(*counts), None if decays is None else (_f32 * T)(*[float(x) for x in decays]),
            _type(grads[0], "grads") if T else 0, copy_type,
            None if coefficient is None else _ptr(coefficient, torch.float32, 1, "coefficient"))


def nuq_adamw_step(ws, grads, ms, vs, decays, alpha: float, beta1: float, beta2: float, eps: float, t: int,
                   coefficient: torch.Tensor | None = None, copies=None) -> None:
    """Step t (1, 2, ...) of AdamW on lists of tensors: weights and both moments fp32, in place; copies: the weights in 16 bits."""
    code = _calls.adamw_step(ws, grads, ms, vs, decays, alpha, beta1, beta2, eps, t, coefficient, copies)
    if code is not None:
        return _check("nuq_adamw_step", code)
    w, g, counts, copy, n, decay, g_type, copy_type, c = _step_arguments(ws, grads, decays, coefficient, copies)
    m, _ = _tensors(ms, "ms", counts, torch.float32)
    v, _ = _tensors(vs, "vs", counts, torch.float32)
    _check("nuq_adamw_step",
           _lib.nuq_adamw_step(len(counts), w, g, m, v, copy, n, decay, g_type, copy_type, float(alpha), float(beta1),
                               float(beta2), float(eps), t, c, _stream()))


def nuq_state_blocks(n: int) -> int:
    return _lib.nuq_state_blocks(n)


def nuq_adamw_step_coded(ws, grads, ms, vs, scales, decays, alpha: float, beta1: float, beta2: float, eps: float, t: int,
                         coefficient: torch.Tensor | None = None, copies=None) -> None:
    """nuq_adamw_step with moments in 8 bits: ms float8_e4m3fn, vs uint8, scales fp32, two per block of STATE_BLOCK elements."""
    code = _calls.adamw_step_coded(ws, grads, ms, vs, scales, decays, alpha, beta1, beta2, eps, t, coefficient, copies)
    if code is not None:
        return _check("nuq_adamw_step_coded", code)
    w, g, counts, copy, n, decay, g_type, copy_type, c = _step_arguments(ws, grads, decays, coefficient, copies)
    m, _ = _tensors(ms, "ms", counts, torch.float8_e4m3fn)
    v, _ = _tensors(vs, "vs", counts, torch.uint8)
    s, _ = _tensors(scales, "scales", [2 * nuq_state_blocks(x) for x in counts], torch.float32)
    _check("nuq_adamw_step_coded",
           _lib.nuq_adamw_step_coded(len(counts), w, g, m, v, s, copy, n, decay, g_type, copy_type, float(alpha), float(beta1),
                                     float(beta2), float(eps), t, c, _stream()))


def nuq_adamw_state_values(m_codes: torch.Tensor, v_codes: torch.Tensor, scales: torch.Tensor, m: torch.Tensor,
                           v: torch.Tensor) -> None:
    """m, v <- the values that the codes of one tensor (or of several, each padded to whole blocks) stand for, fp32."""
    code = _calls.adamw_state_values(m_codes, v_codes, scales, m, v)
    if code is not None:
        return _check("nuq_adamw_state_values", code)
    n = m_codes.numel()
    if v_codes.numel() != n or m.numel() != n or v.numel() != n:
        raise ValueError("codes and values of one length are needed")
    _check("nuq_adamw_state_values",
           _lib.nuq_adamw_state_values(_ptr(m_codes, torch.float8_e4m3fn), _ptr(v_codes, torch.uint8),
                                       _ptr(scales, torch.float32, 2 * nuq_state_blocks(n), "scales"), n,
                                       _ptr(m, torch.float32), _ptr(v, torch.float32), _stream()))


def _rows(t: torch.Tensor, dtype: torch.dtype, rows: int, hidden: int, what: str) -> tuple[int, int]:
    """(address, row stride) of a tensor [..., hidden] as `rows` rows whose elements stand one after the other."""
    if t.dtype is not dtype:
        raise ValueError("%s: expected dtype %s, got %s" % (what, dtype, t.dtype))
    if t.dim() < 1 or t.shape[-1] != hidden or t.numel() != rows * hidden:
        raise ValueError("%s: expected %d rows of %d, got %s" % (what, rows, hidden, tuple(t.shape)))
    if t.dim() != 2:
        try:
            t = t.view(-1, hidden)
        except RuntimeError:
            raise ValueError("%s: its rows do not stand at one stride" % what) from None
    if not _on_device(t) or (hidden > 1 and t.stride(1) != 1):
        raise ValueError("%s: expected a device tensor with contiguous rows" % what)
    return t.data_ptr(), t.stride(0)


def _vector(t: torch.Tensor | None, dtype: torch.dtype, hidden: int, what: str) -> int:
    if t is not None and t.numel() != hidden:
        raise ValueError("%s holds %d elements, %d are needed" % (what, t.numel(), hidden))
    return _ptr(t, dtype, 0, what)


def _weight_dtype(x: torch.Tensor, *vectors) -> torch.dtype:
    for t in vectors:
        if t is not None:
            if t.dtype not in (torch.float32, x.dtype):
                raise ValueError("weight and bias: expected float32 or %s, got %s" % (x.dtype, t.dtype))
            return t.dtype
    return torch.float32


def nuq_layer_norm_forward(x: torch.Tensor, residual: torch.Tensor | None, weight: torch.Tensor | None,
                           bias: torch.Tensor | None, eps: float, total: torch.Tensor | None, y: torch.Tensor,
                           mean: torch.Tensor | None, rstd: torch.Tensor | None) -> None:
    """y <- layer norm of the rows of x [..., hidden], or of total <- x + residual; mean, rstd: a value per row, for backward."""
    code = _calls.layer_norm_forward(x, residual, weight, bias, eps, total, y, mean, rstd)
    if code is not None:
        return _check("nuq_layer_norm_forward", code)
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x: expected rows of one element or more")
    hidden, dtype, kind = x.shape[-1], x.dtype, _weight_dtype(x, weight, bias)
    rows = x.numel() // hidden
    if (residual is None) != (total is None):
        raise ValueError("residual and total: both or neither")
    none = (0, 0)
    px, ldx = _rows(x, dtype, rows, hidden, "x")
    pr, ldr = _rows(residual, dtype, rows, hidden, "residual") if residual is not None else none
    pt, ldt = _rows(total, dtype, rows, hidden, "total") if total is not None else none
    py, ldy = _rows(y, dtype, rows, hidden, "y")
    _check("nuq_layer_norm_forward",
           _lib.nuq_layer_norm_forward(px, ldx, pr, ldr, _vector(weight, kind, hidden, "weight"), _vector(bias, kind, hidden, "bias"),
                                       rows, hidden, float(eps), _type(x, "x"), _TYPES[kind], pt, ldt, py, ldy,
                                       _vector(mean, torch.float32, rows, "mean"), _vector(rstd, torch.float32, rows, "rstd"),
                                       _stream()))


def nuq_layer_norm_workspace_bytes(rows: int, hidden: int) -> int:
    return _lib.nuq_layer_norm_workspace_bytes(rows, hidden)


def nuq_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor | None, mean: torch.Tensor,
                            rstd: torch.Tensor, add: torch.Tensor | None, dx: torch.Tensor, dweight: torch.Tensor | None,
                            dbias: torch.Tensor | None, workspace: torch.Tensor | None) -> None:
    """dx <- the gradient of the rows x (the forward's total where it had one), plus add; dweight, dbias <- theirs."""
    code = _calls.layer_norm_backward(dy, x, weight, mean, rstd, add, dx, dweight, dbias, workspace)
    if code is not None:
        return _check("nuq_layer_norm_backward", code)
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x: expected rows of one element or more")
    hidden, dtype, kind = x.shape[-1], x.dtype, _weight_dtype(x, weight, dweight, dbias)
    rows = x.numel() // hidden
    pg, ldg = _rows(dy, dtype, rows, hidden, "dy")
    px, ldx = _rows(x, dtype, rows, hidden, "x")
    pa, lda = _rows(add, dtype, rows, hidden, "add") if add is not None else (0, 0)
    pd, ldd = _rows(dx, dtype, rows, hidden, "dx")
    _check("nuq_layer_norm_backward",
           _lib.nuq_layer_norm_backward(pg, ldg, px, ldx, _vector(weight, kind, hidden, "weight"),
                                        _vector(mean, torch.float32, rows, "mean"), _vector(rstd, torch.float32, rows, "rstd"),
                                        pa, lda, rows, hidden, _type(x, "x"), _TYPES[kind], pd, ldd,
                                        _vector(dweight, kind, hidden, "dweight"), _vector(dbias, kind, hidden, "dbias"),
                                        _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
                                        _stream()))


# ------------------------------------------ dropout, norms around the residual sum

NO_NORM, LAYER_NORM, RMS_NORM = 0, 1, 2
RESIDUAL_NORM_MAX_HIDDEN = 16384


def _step(step: torch.Tensor | None) -> int:
    return _ptr(step, torch.int64, 0 if step is None else 1, "step")


def _maybe_rows(t: torch.Tensor | None, like: torch.Tensor, what: str) -> tuple[int, int]:
    hidden = like.shape[-1]
    return (0, 0) if t is None else _rows(t, like.dtype, like.numel() // hidden, hidden, what)


def _some_rows(x: torch.Tensor) -> None:
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x: expected rows of one element or more")


def nuq_dropout(x: torch.Tensor, residual: torch.Tensor | None, p: float, seed: int, step: torch.Tensor | None,
                y: torch.Tensor) -> None:
    """y <- x [..., hidden] where kept, with its scale, 0 elsewhere, plus residual; the mask follows from seed, *step and the place."""
    code = _calls.dropout(x, residual, p, seed, step, y)
    if code is not None:
        return _check("nuq_dropout", code)
    _some_rows(x)
    hidden = x.shape[-1]
    _check("nuq_dropout",
           _lib.nuq_dropout(*_maybe_rows(x, x, "x"), *_maybe_rows(residual, x, "residual"), x.numel() // hidden, hidden, _type(x, "x"),
                            float(p), seed & (1 << 64) - 1, _step(step), *_maybe_rows(y, x, "y"), _stream()))


def nuq_residual_norm_forward(x: torch.Tensor, residual: torch.Tensor | None, inner: int, inner_weight: torch.Tensor | None,
                              inner_bias: torch.Tensor | None, gate: torch.Tensor | None, outer: int,
                              outer_weight: torch.Tensor | None, outer_bias: torch.Tensor | None, eps: float, scale: float,
                              residual_scale: float, p: float, seed: int, step: torch.Tensor | None, total: torch.Tensor,
                              y: torch.Tensor | None, stats: torch.Tensor | None) -> None:
    """total <- residual_scale residual + scale drop(gate norm(x)), y <- norm(total); stats [4, rows]: what backward needs of the norms."""
    code = _calls.residual_norm_forward(x, residual, inner, inner_weight, inner_bias, gate, outer, outer_weight, outer_bias, eps, scale,
                                        residual_scale, p, seed, step, total, y, stats)
    if code is not None:
        return _check("nuq_residual_norm_forward", code)
    _some_rows(x)
    hidden = x.shape[-1]
    rows = x.numel() // hidden
    vectors = {"inner_weight": inner_weight, "inner_bias": inner_bias, "gate": gate, "outer_weight": outer_weight, "outer_bias": outer_bias}
    kind = _weight_dtype(x, *vectors.values())
    w1, b1, g, w2, b2 = (_vector(v, kind, hidden, name) for name, v in vectors.items())
    px, ldx = _maybe_rows(x, x, "x")
    _check("nuq_residual_norm_forward",
           _lib.nuq_residual_norm_forward(px, ldx, *_maybe_rows(residual, x, "residual"), inner, w1, b1, g, outer, w2, b2, rows, hidden,
                                          float(eps), float(scale), float(residual_scale), float(p), seed & (1 << 64) - 1, _step(step),
                                          _type(x, "x"), _TYPES[kind], *_maybe_rows(total, x, "total"), *_maybe_rows(y, x, "y"),
                                          _vector(stats, torch.float32, 4 * rows, "stats"), _stream()))


def nuq_residual_norm_workspace_bytes(rows: int, hidden: int) -> int:
    return _lib.nuq_residual_norm_workspace_bytes(rows, hidden)


def nuq_residual_norm_backward(dy: torch.Tensor | None, dtotal: torch.Tensor | None, x: torch.Tensor, total: torch.Tensor | None,
                               inner: int, inner_weight: torch.Tensor | None, inner_bias: torch.Tensor | None,
                               gate: torch.Tensor | None, outer: int, outer_weight: torch.Tensor | None, scale: float,
                               residual_scale: float, p: float, seed: int, step: torch.Tensor | None, stats: torch.Tensor,
                               dx: torch.Tensor, dresidual: torch.Tensor | None, dinner_weight: torch.Tensor | None,
                               dinner_bias: torch.Tensor | None, dgate: torch.Tensor | None, douter_weight: torch.Tensor | None,
                               douter_bias: torch.Tensor | None, workspace: torch.Tensor | None) -> None:
    """dx, dresidual <- the gradients of branch and stream from those of y and total; the others <- those of the vectors."""
    code = _calls.residual_norm_backward(dy, dtotal, x, total, inner, inner_weight, inner_bias, gate, outer, outer_weight, scale,
                                         residual_scale, p, seed, step, stats, dx, dresidual, dinner_weight, dinner_bias, dgate,
                                         douter_weight, douter_bias, workspace)
    if code is not None:
        return _check("nuq_residual_norm_backward", code)
    _some_rows(x)
    hidden = x.shape[-1]
    rows = x.numel() // hidden
    vectors = {"inner_weight": inner_weight, "inner_bias": inner_bias, "gate": gate, "outer_weight": outer_weight,
               "dinner_weight": dinner_weight, "dinner_bias": dinner_bias, "dgate": dgate, "douter_weight": douter_weight,
               "douter_bias": douter_bias}
    kind = _weight_dtype(x, *vectors.values())
    w1, b1, g, w2, *gradients = (_vector(v, kind, hidden, name) for name, v in vectors.items())
    px, ldx = _maybe_rows(x, x, "x")
    _check("nuq_residual_norm_backward",
           _lib.nuq_residual_norm_backward(*_maybe_rows(dy, x, "dy"), *_maybe_rows(dtotal, x, "dtotal"), px, ldx,
                                           *_maybe_rows(total, x, "total"), inner, w1, b1, g, outer, w2, rows, hidden, float(scale),
                                           float(residual_scale), float(p), seed & (1 << 64) - 1, _step(step), _type(x, "x"),
                                           _TYPES[kind], _vector(stats, torch.float32, 4 * rows, "stats"), *_maybe_rows(dx, x, "dx"),
                                           *_maybe_rows(dresidual, x, "dresidual"), *gradients, _ptr(workspace),
                                           0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))


# ------------------------------------------ the loss of a language model

def _loss_rows(x: torch.Tensor, weight: torch.Tensor):
    """(x's address and stride, weight's, rows, hidden, vocabulary, type)"""
    _some_rows(x)
    if weight.dim() != 2 or weight.shape[0] < 1:
        raise ValueError("weight: expected rows of the vocabulary, got %s" % (tuple(weight.shape),))
    hidden = x.shape[-1]
    return (*_maybe_rows(x, x, "x"), *_rows(weight, x.dtype, weight.shape[0], hidden, "weight"), x.numel() // hidden, hidden,
            weight.shape[0], _type(x, "x"))


def _targets(target: torch.Tensor, rows: int) -> int:
    if target.numel() != rows:
        raise ValueError("target holds %d elements, %d are needed" % (target.numel(), rows))
    return _ptr(target, torch.int64, 0, "target")


def nuq_linear_cross_entropy_workspace_bytes(x: torch.Tensor, weight: torch.Tensor, backward: bool) -> int:
    return _lib.nuq_linear_cross_entropy_workspace_bytes(*_loss_rows(x, weight), int(backward))


def nuq_linear_cross_entropy_forward(x: torch.Tensor, weight: torch.Tensor, target: torch.Tensor, ignore: int, smoothing: float,
                                     loss: torch.Tensor | None, lse: torch.Tensor, mean: torch.Tensor | None,
                                     workspace: torch.Tensor) -> None:
    """loss, lse <- softmax cross entropy of x weight^T and its log-sum-exp, per row; mean <- the mean loss, 1 / rows that count."""
    code = _calls.linear_cross_entropy_forward(x, weight, target, ignore, smoothing, loss, lse, mean, workspace)
    if code is not None:
        return _check("nuq_linear_cross_entropy_forward", code)
    shape = _loss_rows(x, weight)
    rows = shape[4]
    _check("nuq_linear_cross_entropy_forward",
           _lib.nuq_linear_cross_entropy_forward(*shape, _targets(target, rows), ignore, float(smoothing),
                                                 _vector(loss, torch.float32, rows, "loss"), _vector(lse, torch.float32, rows, "lse"),
                                                 _vector(mean, torch.float32, 2, "mean"), _ptr(workspace),
                                                 workspace.numel() * workspace.element_size(), _stream()))


def nuq_linear_cross_entropy_backward(x: torch.Tensor, weight: torch.Tensor, target: torch.Tensor, ignore: int, smoothing: float,
                                      lse: torch.Tensor, grad: torch.Tensor, mean: torch.Tensor | None, dx: torch.Tensor | None,
                                      dweight: torch.Tensor | None, workspace: torch.Tensor) -> None:
    """dx, dweight <- the gradients of rows and weights; grad: of the loss, one number or one per row, times mean[1] where given."""
    code = _calls.linear_cross_entropy_backward(x, weight, target, ignore, smoothing, lse, grad, mean, dx, dweight, workspace)
    if code is not None:
        return _check("nuq_linear_cross_entropy_backward", code)
    shape = _loss_rows(x, weight)
    rows, hidden, vocab = shape[4:7]
    if grad.numel() not in (1, rows):
        raise ValueError("grad holds %d elements, 1 or %d are needed" % (grad.numel(), rows))
    pw, ldw = _rows(dweight, x.dtype, vocab, hidden, "dweight") if dweight is not None else (0, 0)
    _check("nuq_linear_cross_entropy_backward",
           _lib.nuq_linear_cross_entropy_backward(*shape, _targets(target, rows), ignore, float(smoothing),
                                                  _vector(lse, torch.float32, rows, "lse"), _ptr(grad, torch.float32, 0, "grad"),
                                                  int(grad.numel() != 1), _vector(mean, torch.float32, 2, "mean"),
                                                  *_maybe_rows(dx, x, "dx"), pw, ldw, _ptr(workspace),
                                                  workspace.numel() * workspace.element_size(), _stream()))


def nuq_last_error_flags() -> int:
    flags = ctypes.c_uint32(0)
    _check("nuq_last_error_flags", _lib.nuq_last_error_flags(ctypes.byref(flags), _stream()))
    return flags.value


# ------------------------------------------------------------ measurement aid

T_NORMS, T_QUANTIZE, T_ENCODE, T_QUANTIZE_ENCODE, T_DECODE = 1, 2, 3, 4, 5


def nuq_encode_shape(mode: int, K: int, d: int, bucket: int, s: int, sync_stride: int, levels=None,
                     norm_kind: int = NORM_L2) -> tuple[int, int, int, int]:
    """(threads per bucket, nonzeros its list holds, words of its string's buffer, words put together at once where the list
    does not hold the nonzeros) of the ERC encoders' main kernel; mode 0: main levels, 1: nuq_encode, 2: a level table."""
    shape = (_u32 * 4)()
    table = (ctypes.c_float * (s + 2))(*levels) if mode == 2 else None
    _check("nuq_encode_shape", _lib.nuq_encode_shape(mode, K, d, bucket, s, sync_stride, table, norm_kind, shape))
    return tuple(shape)


def nuq_decode_tile(K: int, d: int, bucket: int, s: int, sync_stride: int, table: bool = False, update: int = 0) -> int:
    return _lib.nuq_decode_tile(K, d, bucket, s, sync_stride, int(table), update)


def nuq_timing_begin(max_launches: int) -> None:
    _check("nuq_timing_begin", _lib.nuq_timing_begin(max_launches))


def nuq_timing_collect(cap: int = 4096) -> list[tuple[int, float]]:
    """[(entry point id, milliseconds)] for the launches bracketed since nuq_timing_begin."""
    ms = (ctypes.c_float * cap)()
    entry = (ctypes.c_int32 * cap)()
    count = ctypes.c_uint32(0)
    _check("nuq_timing_collect", _lib.nuq_timing_collect(ms, entry, cap, ctypes.byref(count)))
    return [(entry[i], ms[i]) for i in range(count.value)]
