"""ctypes marshalling for the C ABI declared in include/qkvcard.h (same names, same order)."""
import contextlib
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_NAME = "libqkvcard.so"

STATUS_BAD_BITS = 0x1
STATUS_BAD_COUNTS = 0x2
STATUS_BAD_HEADER = 0x4
STATUS_BAD_ORDER = 0x8
STATUS_BAD_PAGE = 0x10
STATUS_BAD_ROW = 0x20
STATUS_NO_PAGES = 0x40
FLAG_KEYS_PER_CHANNEL = 0x1


class QkvError(RuntimeError):
    def __init__(self, code, where):
        super().__init__("%s: %s (%d)" % (where, error_string(code), code))
        self.code = code


class Desc(ctypes.Structure):
    """qkv_desc_t."""
    _fields_ = [
        ("layers", ctypes.c_int32),
        ("kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("group_size", ctypes.c_int32),
        ("tokens", ctypes.c_int64),
        ("model_id", ctypes.c_uint64),
        ("sender_id", ctypes.c_uint64),
        ("position_offset", ctypes.c_int64),
    ]

    @classmethod
    def make(cls, layers, kv_heads, tokens, head_dim, group_size, model_id=0, sender_id=0, position_offset=0):
        return cls(layers, kv_heads, head_dim, group_size, tokens, model_id, sender_id, position_offset)


class Controller(ctypes.Structure):
    """qkv_controller_t: the 512 parameters of the 6 -> 64 -> 1 network."""
    _fields_ = [("w1", ctypes.c_float * 6 * 64), ("b1", ctypes.c_float * 64), ("w2", ctypes.c_float * 64)]

    @classmethod
    def make(cls, w1, b1, w2):
        """w1 [64, 6], b1 [64], w2 [64]: host float32 tensors or arrays."""
        c = cls()
        flat = [float(x) for x in torch.as_tensor(w1, dtype=torch.float32).reshape(-1).tolist()]
        if len(flat) != 384 or len(b1) != 64 or len(w2) != 64:
            raise ValueError("controller parameters must be w1 [64, 6], b1 [64], w2 [64]")
        ctypes.memmove(c.w1, (ctypes.c_float * 384)(*flat), 384 * 4)
        ctypes.memmove(c.b1, (ctypes.c_float * 64)(*[float(x) for x in torch.as_tensor(b1, dtype=torch.float32).tolist()]), 256)
        ctypes.memmove(c.w2, (ctypes.c_float * 64)(*[float(x) for x in torch.as_tensor(w2, dtype=torch.float32).tolist()]), 256)
        return c


class Inject(ctypes.Structure):
    """qkv_inject_t."""
    _fields_ = [
        ("layer_begin", ctypes.c_int32),
        ("layer_count", ctypes.c_int32),
        ("k_layers", ctypes.POINTER(ctypes.c_void_p)),
        ("v_layers", ctypes.POINTER(ctypes.c_void_p)),
        ("head_stride", ctypes.c_int64),
        ("token_stride", ctypes.c_int64),
        ("rope_base", ctypes.c_double),
        ("rope_delta", ctypes.c_int64),
        ("keys_per_channel", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
    ]


class _InjectByAddress(ctypes.Structure):
    """qkv_inject_t with the tables' addresses as numbers."""
    _fields_ = [(name, ctypes.c_size_t if name in ("k_layers", "v_layers") else kind) for name, kind in Inject._fields_]


class Pages(ctypes.Structure):
    """qkv_pages_t, and the tensors it points to, which it keeps alive."""
    _fields_ = [
        ("layers", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("page_tokens", ctypes.c_int32),
        ("value_type", ctypes.c_int32), ("pages", ctypes.c_int32), ("rows", ctypes.c_int32), ("row_pages", ctypes.c_int32),
        ("k_layers", ctypes.POINTER(ctypes.c_void_p)), ("v_layers", ctypes.POINTER(ctypes.c_void_p)),
        ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
        ("table_dev", ctypes.c_void_p), ("lens_dev", ctypes.c_void_p), ("refs_dev", ctypes.c_void_p),
    ]

    @classmethod
    def make(cls, k_layers, v_layers, table, lens, refs=None):
        """k_layers, v_layers: lists of device float16 or bfloat16 tensors (views are fine) [pages, kv_heads, page_tokens, head_dim], rows
        contiguous, all with the same strides; table: device int32 [rows, row_pages]; lens: device int32 [rows]; refs: device int32 [pages]
        (needed by pages_reserve, pages_fork, pages_free and pages_compact)."""
        count = len(k_layers)
        if count < 1 or count != len(v_layers):
            raise ValueError("k_layers and v_layers must be lists of the same, non-zero length")
        first = k_layers[0]
        if first.dtype not in _VALUE_TYPES:
            raise ValueError("pages must be float16 or bfloat16")
        for t in (*k_layers, *v_layers):
            if t.dim() != 4 or t.dtype != first.dtype or t.shape != first.shape or t.device != first.device or not t.is_cuda:
                raise ValueError("layer tensors must be device tensors [pages, kv_heads, page_tokens, head_dim] of one type, shape and device")
            if t.stride() != first.stride() or t.stride(3) != 1:
                raise ValueError("layer tensors must share their strides and have contiguous rows")
        for t, shape, name in ((table, None, "table"), (lens, (table.shape[0],), "lens"), (refs, (first.shape[0],), "refs")):
            if t is None and name == "refs":
                continue
            _dev_ptr(t, torch.int32, name)
            if t.device != first.device:
                raise ValueError("%s must live on the pages' device" % name)
            if t.dim() != 2 if shape is None else tuple(t.shape) != shape:
                raise ValueError("%s has the wrong shape" % name)
        pointers = (ctypes.c_void_p * (2 * count))(*[t.data_ptr() for t in (*k_layers, *v_layers)])
        values = ctypes.cast(ctypes.addressof(pointers) + 8 * count, ctypes.POINTER(ctypes.c_void_p))
        p = cls(count, first.shape[1], first.shape[3], first.shape[2], _VALUE_TYPES[first.dtype], first.shape[0], table.shape[0], table.shape[1],
                ctypes.cast(pointers, ctypes.POINTER(ctypes.c_void_p)), values, first.stride(0), first.stride(1), first.stride(2),
                table.data_ptr(), lens.data_ptr(), None if refs is None else refs.data_ptr())
        p.tensors = (list(k_layers), list(v_layers), table, lens, refs, pointers)
        p.dtype, p.device = first.dtype, first.device
        return p


class Rows(ctypes.Structure):
    """qkv_rows_t."""
    _fields_ = [
        ("k_dev", ctypes.c_size_t), ("v_dev", ctypes.c_size_t), ("tokens", ctypes.c_int64),
        ("layer_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
        ("starts_dev", ctypes.c_size_t), ("layer_begin", ctypes.c_int32), ("layer_count", ctypes.c_int32),
    ]


class PagedQuery(ctypes.Structure):
    """qkv_paged_query_t."""
    _fields_ = [
        ("q_dev", ctypes.c_size_t), ("q_token_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64), ("tokens", ctypes.c_int64),
        ("starts_dev", ctypes.c_size_t), ("out_dev", ctypes.c_size_t), ("lse_dev", ctypes.c_size_t), ("prior_out_dev", ctypes.c_size_t),
        ("prior_lse_dev", ctypes.c_size_t), ("workspace_dev", ctypes.c_size_t), ("workspace_bytes", ctypes.c_uint64),
        ("status_dev", ctypes.c_size_t), ("layer", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("window", ctypes.c_int32),
        ("sinks", ctypes.c_int32), ("softmax_scale", ctypes.c_float), ("reserved", ctypes.c_int32),
    ]


_VALUE_TYPES = {torch.float16: 0, torch.bfloat16: 1}

_pointer_tables = [ctypes.c_void_p * (2 * count) for count in range(5)]

_lib = None
_inject_by_address = None         # qkv_inject_layers for an _InjectByAddress; set with _lib


def lib_path():
    return os.path.join(_HERE, _LIB_NAME)


def lib():
    """The loaded library.  Built once by paper_2605_03884_amd.build if it is not there; never replaced by a fallback."""
    global _lib, _inject_by_address
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        from . import build as _build
        _build.build()
    L = ctypes.CDLL(path)
    i64p = ctypes.POINTER(ctypes.c_int64)
    vp = ctypes.c_void_p
    L.qkv_version.restype = ctypes.c_int
    L.qkv_version.argtypes = []
    L.qkv_error_string.restype = ctypes.c_char_p
    L.qkv_error_string.argtypes = [ctypes.c_int]
    L.qkv_card_bytes.restype = ctypes.c_int
    L.qkv_card_bytes.argtypes = [ctypes.POINTER(Desc), i64p, ctypes.POINTER(ctypes.c_uint64)]
    L.qkv_budget_counts.restype = ctypes.c_int
    L.qkv_budget_counts.argtypes = [ctypes.c_int64, ctypes.c_double, i64p]
    L.qkv_assign_bits.restype = ctypes.c_int
    L.qkv_assign_bits.argtypes = [vp, ctypes.c_int64, ctypes.c_double, vp, i64p, vp]
    L.qkv_assign_plan.restype = ctypes.c_int
    L.qkv_assign_plan.argtypes = [ctypes.POINTER(Desc), vp, ctypes.c_double, vp, i64p, vp, ctypes.c_uint64, vp]
    L.qkv_assign_quantize_pack.restype = ctypes.c_int
    L.qkv_assign_quantize_pack.argtypes = [ctypes.POINTER(Desc), vp, vp, vp, ctypes.c_double, vp, i64p, vp, ctypes.c_uint64, vp]
    L.qkv_controller_scores.restype = ctypes.c_int
    L.qkv_controller_scores.argtypes = [vp, ctypes.c_int64, ctypes.POINTER(Controller), vp, vp]
    L.qkv_assign_bits_greedy.restype = ctypes.c_int
    L.qkv_assign_bits_greedy.argtypes = [vp, ctypes.c_int64, ctypes.c_double, vp, vp, vp]
    L.qkv_count_bits.restype = ctypes.c_int
    L.qkv_count_bits.argtypes = [vp, ctypes.c_int64, i64p, vp]
    L.qkv_quantize_pack.restype = ctypes.c_int
    L.qkv_quantize_pack.argtypes = [ctypes.POINTER(Desc), vp, vp, vp, i64p, vp, ctypes.c_uint64, vp]
    L.qkv_card_plan.restype = ctypes.c_int
    L.qkv_card_plan.argtypes = [ctypes.POINTER(Desc), vp, i64p, vp, ctypes.c_uint64, vp]
    L.qkv_card_fill.restype = ctypes.c_int
    L.qkv_card_fill.argtypes = [ctypes.POINTER(Desc), vp, vp, i64p, vp, ctypes.c_uint64, vp]
    L.qkv_inject_layers.restype = ctypes.c_int
    L.qkv_inject_layers.argtypes = [vp, ctypes.c_uint64, ctypes.POINTER(Desc), ctypes.POINTER(Inject), vp, vp]
    inject = L["qkv_inject_layers"]                # the same entry point, a prototype of its own
    inject.restype = ctypes.c_int
    inject.argtypes = [vp, ctypes.c_uint64, ctypes.POINTER(Desc), ctypes.POINTER(_InjectByAddress), vp, vp]
    L.qkv_quantize_pack_kc.restype = ctypes.c_int
    L.qkv_quantize_pack_kc.argtypes = [ctypes.POINTER(Desc), vp, vp, vp, i64p, vp, ctypes.c_uint64, vp]
    L.qkv_unpack_dequant_kc.restype = ctypes.c_int
    L.qkv_unpack_dequant_kc.argtypes = [vp, ctypes.c_uint64, ctypes.POINTER(Desc), vp, vp, vp, vp]
    L.qkv_requantize.restype = ctypes.c_int
    L.qkv_requantize.argtypes = [vp, ctypes.c_uint64, ctypes.POINTER(Desc), vp, i64p, vp, ctypes.c_uint64, vp, vp]
    L.qkv_unpack_dequant.restype = ctypes.c_int
    L.qkv_unpack_dequant.argtypes = [vp, ctypes.c_uint64, ctypes.POINTER(Desc), vp, vp, vp, vp]
    L.qkv_card_attend_workspace.restype = ctypes.c_int
    L.qkv_card_attend_workspace.argtypes = [ctypes.POINTER(Desc), ctypes.c_int32, ctypes.POINTER(ctypes.c_uint64)]
    L.qkv_card_attend.restype = ctypes.c_int
    L.qkv_card_attend.argtypes = [vp, ctypes.c_uint64, ctypes.POINTER(Desc), vp, ctypes.c_int32, ctypes.c_float, vp, vp,
                                  vp, ctypes.c_uint64, vp, vp]
    L.qkv_card_attend_kc.restype = ctypes.c_int
    L.qkv_card_attend_kc.argtypes = [vp, ctypes.c_uint64, ctypes.POINTER(Desc), vp, ctypes.c_int32, ctypes.c_float, vp, vp,
                                  vp, ctypes.c_uint64, vp, vp]
    L.qkv_card_attend_static.restype = ctypes.c_int
    L.qkv_card_attend_static.argtypes = [vp, ctypes.c_uint64, ctypes.POINTER(Desc), vp, ctypes.c_int32, ctypes.c_float, vp, vp,
                                         vp, vp]
    pages, bytes_out = ctypes.POINTER(Pages), ctypes.POINTER(ctypes.c_uint64)
    for name, args in (("pages_reserve", [pages, vp, vp, vp]),
                       ("pages_append", [pages, ctypes.POINTER(Rows), vp, vp]),
                       ("pages_fork", [pages, vp, vp, ctypes.c_int32, vp, vp]),
                       ("pages_free", [pages, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp, vp]),
                       ("pages_compact_workspace", [pages, bytes_out]),
                       ("pages_compact", [pages, vp, vp, ctypes.c_uint64, vp, vp]),
                       ("paged_attend_workspace", [pages, ctypes.c_int32, bytes_out]),
                       ("paged_attend", [pages, ctypes.POINTER(PagedQuery), vp]),
                       ("paged_prompt_workspace", [pages, ctypes.c_int32, ctypes.c_int64, bytes_out]),
                       ("paged_prompt", [pages, ctypes.POINTER(PagedQuery), vp])):
        entry = getattr(L, "qkv_" + name)
        entry.restype, entry.argtypes = ctypes.c_int, args
    L.qkv_card_peek.restype = ctypes.c_int
    L.qkv_card_peek.argtypes = [vp, ctypes.c_uint64, ctypes.POINTER(Desc), i64p, ctypes.POINTER(ctypes.c_float),
                                ctypes.POINTER(ctypes.c_uint32), vp]
    L.qkv_card_flags.restype = ctypes.c_int
    L.qkv_card_flags.argtypes = [vp, ctypes.c_uint64, ctypes.POINTER(ctypes.c_uint32), vp]
    _inject_by_address = inject                    # before _lib: another thread that finds _lib set finds this too
    _lib = L
    return L


def _check(rc, where):
    if rc != 0:
        raise QkvError(rc, where)


_Counts = ctypes.c_int64 * 4


def _counts(counts):
    return _Counts(*map(int, counts))


# The current stream's handle without the object torch.cuda.current_stream() builds (2.9 us of a call's 8), and the current device without
# torch.cuda.current_device()'s look from Python whether CUDA is set up (0.2 us), which the native call makes by itself: in a forked child
# too it asks torch's initialization, which refuses.  Not part of torch's public interface: where a torch lacks them, the public calls are made.
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _stream(stream):
    """The stream's handle; the current stream of the current device without one."""
    if stream is None:
        if _current_raw_stream is None:
            return torch.cuda.current_stream().cuda_stream
        return _current_raw_stream(_current_device())
    return stream.cuda_stream


def _scratch(nbytes, device, stream):
    """Device memory for a call that brings none of its own.  It is given back when the call returns, so it is taken from the memory of the stream
    the call runs on: whoever gets it next is queued behind the call's work, and the call behind whoever had it before."""
    with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _dev_ptr(t, dtype=None, name="tensor"):
    if not t.is_cuda:
        raise ValueError("%s must live in device memory" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s must be %s" % (name, dtype))
    return t.data_ptr()


def _optional_ptr(t, dtype=None, name="tensor"):
    return None if t is None else _dev_ptr(t, dtype, name)


def version():
    return lib().qkv_version()


def error_string(code):
    return lib().qkv_error_string(int(code)).decode()


def card_bytes(desc, counts):
    out = ctypes.c_uint64(0)
    _check(lib().qkv_card_bytes(ctypes.byref(desc), _counts(counts), ctypes.byref(out)), "qkv_card_bytes")
    return out.value


def budget_counts(tokens, avg_bits_budget):
    out = _Counts()
    _check(lib().qkv_budget_counts(int(tokens), float(avg_bits_budget), out), "qkv_budget_counts")
    return list(out)


def assign_bits(scores, avg_bits_budget, bits=None, stream=None):
    """scores: device float32[T].  Returns (bits device uint8[T], counts list)."""
    T = scores.numel()
    if bits is None:
        bits = torch.empty(T, dtype=torch.uint8, device=scores.device)
    out = _Counts()
    _check(lib().qkv_assign_bits(_dev_ptr(scores, torch.float32, "scores"), T, float(avg_bits_budget),
                                 _dev_ptr(bits, torch.uint8, "bits"), out, _stream(stream)), "qkv_assign_bits")
    return bits, list(out)


def assign_plan(desc, scores, avg_bits_budget, card, bits=None, stream=None):
    """scores: device float32[T]; card: device uint8 buffer (header, tables and pads are written); bits: device
    uint8[T] or None.  Returns the class counts (list)."""
    out = _Counts()
    bp = _optional_ptr(bits, torch.uint8, "bits")
    _check(lib().qkv_assign_plan(ctypes.byref(desc), _dev_ptr(scores, torch.float32, "scores"), float(avg_bits_budget), bp,
                                 out, _dev_ptr(card, torch.uint8, "card"), card.numel(), _stream(stream)),
           "qkv_assign_plan")
    return list(out)


def assign_quantize_pack(desc, k, v, scores, avg_bits_budget, card, bits=None, stream=None):
    """Scores, budget and K/V in; widths (if bits is given) and the whole card out.  Returns the class counts."""
    out = _Counts()
    bp = _optional_ptr(bits, torch.uint8, "bits")
    _check(lib().qkv_assign_quantize_pack(ctypes.byref(desc), _dev_ptr(k, torch.float16, "k"), _dev_ptr(v, torch.float16, "v"),
                                          _dev_ptr(scores, torch.float32, "scores"), float(avg_bits_budget), bp, out,
                                          _dev_ptr(card, torch.uint8, "card"), card.numel(), _stream(stream)),
           "qkv_assign_quantize_pack")
    return list(out)


def controller_scores(features, params, scores=None, stream=None):
    """features: device float32[T, 6]; params: Controller.  Returns scores, device float32[T]."""
    T = features.shape[0]
    if features.dim() != 2 or features.shape[1] != 6:
        raise ValueError("features must be [T, 6]")
    if scores is None:
        scores = torch.empty(T, dtype=torch.float32, device=features.device)
    _check(lib().qkv_controller_scores(_dev_ptr(features, torch.float32, "features"), T, ctypes.byref(params),
                                       _dev_ptr(scores, torch.float32, "scores"), _stream(stream)),
           "qkv_controller_scores")
    return scores


def assign_bits_greedy(scores, avg_bits_budget, bits=None, counts=None, stream=None):
    """scores: device float32[T].  Returns (bits device uint8[T], counts device int64[4]); nothing synchronises."""
    T = scores.numel()
    if bits is None:
        bits = torch.empty(T, dtype=torch.uint8, device=scores.device)
    if counts is None:
        counts = torch.empty(4, dtype=torch.int64, device=scores.device)
    _check(lib().qkv_assign_bits_greedy(_dev_ptr(scores, torch.float32, "scores"), T, float(avg_bits_budget),
                                        _dev_ptr(bits, torch.uint8, "bits"), _dev_ptr(counts, torch.int64, "counts"),
                                        _stream(stream)), "qkv_assign_bits_greedy")
    return bits, counts


def count_bits(bits, stream=None):
    out = _Counts()
    _check(lib().qkv_count_bits(_dev_ptr(bits, torch.uint8, "bits"), bits.numel(), out, _stream(stream)),
           "qkv_count_bits")
    return list(out)


def quantize_pack(desc, k, v, bits, counts, card, stream=None):
    """k, v: device float16 [L, H, T, D]; bits: device uint8[T]; card: device uint8 buffer, written in place."""
    _check(lib().qkv_quantize_pack(ctypes.byref(desc), _dev_ptr(k, torch.float16, "k"), _dev_ptr(v, torch.float16, "v"),
                                   _dev_ptr(bits, torch.uint8, "bits"), _counts(counts),
                                   _dev_ptr(card, torch.uint8, "card"), card.numel(), _stream(stream)),
           "qkv_quantize_pack")
    return card


def quantize_pack_kc(desc, k, v, bits, counts, card, stream=None):
    """quantize_pack for a uniform card with the keys grouped per channel."""
    _check(lib().qkv_quantize_pack_kc(ctypes.byref(desc), _dev_ptr(k, torch.float16, "k"), _dev_ptr(v, torch.float16, "v"),
                                      _dev_ptr(bits, torch.uint8, "bits"), _counts(counts),
                                      _dev_ptr(card, torch.uint8, "card"), card.numel(), _stream(stream)),
           "qkv_quantize_pack_kc")
    return card


def requantize(card_in, desc, bits, counts, card_out, status=None, card_in_nbytes=None, stream=None):
    """The card that quantize_pack would build from unpack_dequant(card_in), at the new widths, card to card.  Where card_in is a buffer
    longer than its card, card_in_nbytes should name the card's own length: the kernel is chosen by it."""
    n = card_in.numel() if card_in_nbytes is None else int(card_in_nbytes)
    sp = _optional_ptr(status, None, "status")
    _check(lib().qkv_requantize(_dev_ptr(card_in, torch.uint8, "card_in"), n, ctypes.byref(desc),
                                _dev_ptr(bits, torch.uint8, "bits"), _counts(counts),
                                _dev_ptr(card_out, torch.uint8, "card_out"), card_out.numel(), sp, _stream(stream)),
           "qkv_requantize")
    return card_out


def card_plan(desc, bits, counts, card, stream=None):
    """First half of quantize_pack: header, tables and pads."""
    _check(lib().qkv_card_plan(ctypes.byref(desc), _dev_ptr(bits, torch.uint8, "bits"), _counts(counts),
                               _dev_ptr(card, torch.uint8, "card"), card.numel(), _stream(stream)), "qkv_card_plan")
    return card


def card_fill(desc, k, v, counts, card, stream=None):
    """Second half of quantize_pack: the K/V rows into a planned card."""
    _check(lib().qkv_card_fill(ctypes.byref(desc), _dev_ptr(k, torch.float16, "k"), _dev_ptr(v, torch.float16, "v"),
                               _counts(counts), _dev_ptr(card, torch.uint8, "card"), card.numel(), _stream(stream)),
           "qkv_card_fill")
    return card


def unpack_dequant(card, expect, k_out, v_out, status=None, card_nbytes=None, stream=None):
    """card: device uint8; k_out, v_out: device float16 [L, H, T, D]; status: device int32[1] or None."""
    n = card.numel() if card_nbytes is None else int(card_nbytes)
    sp = _optional_ptr(status, None, "status")
    _check(lib().qkv_unpack_dequant(_dev_ptr(card, torch.uint8, "card"), n, ctypes.byref(expect),
                                    _dev_ptr(k_out, torch.float16, "k_out"), _dev_ptr(v_out, torch.float16, "v_out"),
                                    sp, _stream(stream)), "qkv_unpack_dequant")
    return k_out, v_out


def unpack_dequant_kc(card, expect, k_out, v_out, status=None, card_nbytes=None, stream=None):
    """unpack_dequant for a uniform card with the keys grouped per channel."""
    n = card.numel() if card_nbytes is None else int(card_nbytes)
    sp = _optional_ptr(status, None, "status")
    _check(lib().qkv_unpack_dequant_kc(_dev_ptr(card, torch.uint8, "card"), n, ctypes.byref(expect),
                                       _dev_ptr(k_out, torch.float16, "k_out"), _dev_ptr(v_out, torch.float16, "v_out"),
                                       sp, _stream(stream)), "qkv_unpack_dequant_kc")
    return k_out, v_out


def inject_layers(card, expect, k_layers, v_layers, layer_begin=0, rope_base=0.0, rope_delta=0, status=None,
                  card_nbytes=None, stream=None, keys_per_channel=False):
    """Layers layer_begin .. layer_begin + len(k_layers) - 1 of the card into per-layer tensors.

    k_layers, v_layers: lists of device float16 tensors (views are fine) of shape [kv_heads, >= tokens, head_dim]
    whose element [h, t, :] is where token t of head h lands: rows contiguous, all layers with the same strides.
    A cache [kv_heads, capacity, head_dim] holding a prefix of P tokens is passed as cache[:, P:P + tokens]."""
    n = card.numel() if card_nbytes is None else int(card_nbytes)
    count = len(k_layers)
    if count != len(v_layers) or count < 1:
        raise ValueError("k_layers and v_layers must be lists of the same, non-zero length")
    strides = k_layers[0].stride()
    heads, tokens, dim, half = expect.kv_heads, expect.tokens, expect.head_dim, torch.float16
    pointers = []
    for tensors in (k_layers, v_layers):
        for t in tensors:
            shape = t.shape
            if t.dtype is not half or len(shape) != 3 or not t.is_cuda:
                raise ValueError("layer tensors must be device float16 [kv_heads, tokens, head_dim]")
            if shape[0] != heads or shape[1] < tokens or shape[2] != dim:
                raise ValueError("layer tensor shape %s does not hold the card's tokens" % (tuple(shape),))
            if t.stride() != strides or strides[2] != 1:
                raise ValueError("layer tensors must share their strides and have contiguous rows")
            pointers.append(t.data_ptr())
    # One table for both, and its address as a number: a receiver makes this call once a layer, and with two arrays behind
    # pointer fields the arguments alone took 0.8 us.
    table = _pointer_tables[count](*pointers) if count < len(_pointer_tables) else (ctypes.c_void_p * (2 * count))(*pointers)
    at = ctypes.addressof(table)
    where = _InjectByAddress(int(layer_begin), count, at, at + 8 * count, strides[0], strides[1], float(rope_base), int(rope_delta),
                             1 if keys_per_channel else 0, 0)
    if _inject_by_address is None:
        lib()
    _check(_inject_by_address(_dev_ptr(card, torch.uint8, "card"), n, expect, where,          # structures themselves: 0.3 us less than by byref()
                              None if status is None else _dev_ptr(status, None, "status"), _stream(stream)), "qkv_inject_layers")


def card_attend_workspace(expect, q_heads):
    out = ctypes.c_uint64(0)
    _check(lib().qkv_card_attend_workspace(ctypes.byref(expect), int(q_heads), ctypes.byref(out)),
           "qkv_card_attend_workspace")
    return out.value


def card_attend(card, expect, q, softmax_scale, out, lse=None, workspace=None, status=None, card_nbytes=None,
                stream=None):
    """card: device uint8; q: device float16 [L, Hq, D]; out: device float32 [L, Hq, D]; lse: float32 [L, Hq]; D = 64, 128 or 256."""
    n = card.numel() if card_nbytes is None else int(card_nbytes)
    q_heads = q.shape[1]
    if workspace is None:
        workspace = _scratch(card_attend_workspace(expect, q_heads), card.device, stream)
    lp = _optional_ptr(lse, torch.float32, "lse")
    sp = _optional_ptr(status, None, "status")
    _check(lib().qkv_card_attend(_dev_ptr(card, torch.uint8, "card"), n, ctypes.byref(expect),
                                 _dev_ptr(q, torch.float16, "q"), int(q_heads), float(softmax_scale),
                                 _dev_ptr(out, torch.float32, "out"), lp, _dev_ptr(workspace, torch.uint8, "workspace"),
                                 workspace.numel(), sp, _stream(stream)), "qkv_card_attend")
    return out, lse


def card_attend_kc(card, expect, q, softmax_scale, out, lse=None, workspace=None, status=None, card_nbytes=None,
                   stream=None):
    """card_attend for a card whose keys are grouped per channel (made by quantize_pack_kc)."""
    n = card.numel() if card_nbytes is None else int(card_nbytes)
    q_heads = q.shape[1]
    if workspace is None:
        workspace = _scratch(card_attend_workspace(expect, q_heads), card.device, stream)
    lp = _optional_ptr(lse, torch.float32, "lse")
    sp = _optional_ptr(status, None, "status")
    _check(lib().qkv_card_attend_kc(_dev_ptr(card, torch.uint8, "card"), n, ctypes.byref(expect),
                                    _dev_ptr(q, torch.float16, "q"), int(q_heads), float(softmax_scale),
                                    _dev_ptr(out, torch.float32, "out"), lp, _dev_ptr(workspace, torch.uint8, "workspace"),
                                    workspace.numel(), sp, _stream(stream)), "qkv_card_attend_kc")
    return out, lse


def card_attend_static(card, expect, q, softmax_scale, out, lse=None, status=None, card_nbytes=None, stream=None):
    """card_attend without a workspace: the partials live in the library's fixed scratch array (no allocation)."""
    n = card.numel() if card_nbytes is None else int(card_nbytes)
    lp = _optional_ptr(lse, torch.float32, "lse")
    sp = _optional_ptr(status, None, "status")
    _check(lib().qkv_card_attend_static(_dev_ptr(card, torch.uint8, "card"), n, ctypes.byref(expect),
                                        _dev_ptr(q, torch.float16, "q"), int(q.shape[1]), float(softmax_scale),
                                        _dev_ptr(out, torch.float32, "out"), lp, sp, _stream(stream)), "qkv_card_attend_static")
    return out, lse


def card_flags(card, card_nbytes=None, stream=None):
    """The header's flags word (0 or FLAG_KEYS_PER_CHANNEL) of a valid card.  Synchronises the stream."""
    n = card.numel() if card_nbytes is None else int(card_nbytes)
    fl = ctypes.c_uint32(0)
    _check(lib().qkv_card_flags(_dev_ptr(card, torch.uint8, "card"), n, ctypes.byref(fl), _stream(stream)),
           "qkv_card_flags")
    return fl.value


def card_peek(card, card_nbytes=None, stream=None):
    """Returns (Desc, counts, avg_bits, status).  Synchronises the stream."""
    n = card.numel() if card_nbytes is None else int(card_nbytes)
    d = Desc()
    counts = _Counts()
    avg = ctypes.c_float(0)
    st = ctypes.c_uint32(0)
    _check(lib().qkv_card_peek(_dev_ptr(card, torch.uint8, "card"), n, ctypes.byref(d), counts, ctypes.byref(avg),
                               ctypes.byref(st), _stream(stream)), "qkv_card_peek")
    return d, list(counts), avg.value, st.value


def _here(pages, stream):
    """The stream's handle; the current stream of the pages' device without one.  Calls go to the current device: it has to be the pages'."""
    if pages.device.index != _current_device():
        raise ValueError("the pages live on %s: make it the current device" % pages.device)
    return _stream(stream)


def _of_pages(t, pages, dtype, shape, name):
    """The address of a contiguous tensor on the pages' device."""
    if t.device != pages.device or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor %s on %s" % (name, dtype, list(shape), pages.device))
    return t.data_ptr()


def _status_of_pages(status, pages):
    if status is None:
        return 0
    if status.device != pages.device or status.numel() < 1 or status.dtype.itemsize != 4:
        raise ValueError("status must be one 32-bit word on %s" % pages.device)
    return status.data_ptr()


def pages_reserve(pages, more, status, stream=None):
    """Room for more[i] (device int32 [rows]; None: 1 each) new tokens in every row; lens are the new lengths afterwards."""
    at = None if more is None else _of_pages(more, pages, torch.int32, (pages.rows,), "more")
    _check(lib().qkv_pages_reserve(pages, at, _status_of_pages(status, pages), _here(pages, stream)), "qkv_pages_reserve")


def pages_append(pages, k, v, layer=0, starts=None, status=None, stream=None):
    """k, v: device tensors of the pages' type [layers, tokens, kv_heads, head_dim] or, of one layer, [tokens, kv_heads, head_dim] (views with
    contiguous rows are fine, both with the same strides) into the pages of layer `layer` and on; starts: device int32 [rows + 1], or None for
    one token a row.  A dense cache [layers, kv_heads, tokens, head_dim] is passed as .transpose(1, 2)."""
    if k.dim() == 3:
        k, v = k.unsqueeze(0), v.unsqueeze(0)
    shape, strides = k.shape, k.stride()
    if len(shape) != 4 or v.shape != shape or v.stride() != strides or strides[3] != 1 or shape[2] != pages.kv_heads or shape[3] != pages.head_dim:
        raise ValueError("k and v must be [layers, tokens, kv_heads, head_dim] with the same strides and contiguous rows")
    if k.dtype is not pages.dtype or v.dtype is not pages.dtype or k.device != pages.device or v.device != pages.device:
        raise ValueError("k and v must have the pages' type and device")
    if shape[1] == 0:
        return
    at = 0 if starts is None else _of_pages(starts, pages, torch.int32, (pages.rows + 1,), "starts")
    rows = Rows(k.data_ptr(), v.data_ptr(), shape[1], strides[0], strides[2], strides[1], at, layer, shape[0])
    _check(lib().qkv_pages_append(pages, rows, _status_of_pages(status, pages), _here(pages, stream)), "qkv_pages_append")


def pages_fork(pages, source, target, status, stream=None):
    """Rows target[i] go on from rows source[i] (device int32 [n])."""
    n = source.numel()
    _check(lib().qkv_pages_fork(pages, _of_pages(source, pages, torch.int32, (n,), "source"), _of_pages(target, pages, torch.int32, (n,), "target"), n,
                                _status_of_pages(status, pages), _here(pages, stream)), "qkv_pages_fork")


def pages_free(pages, rows=None, window=0, sinks=0, status=None, stream=None):
    """Gives back the pages of the rows (device int32 [n]; None: all), with a window only those that are out of sight for good."""
    n = pages.rows if rows is None else rows.numel()
    at = None if rows is None else _of_pages(rows, pages, torch.int32, (n,), "rows")
    _check(lib().qkv_pages_free(pages, at, n, int(window), int(sinks), _status_of_pages(status, pages), _here(pages, stream)), "qkv_pages_free")


def pages_compact_workspace(pages):
    out = ctypes.c_uint64(0)
    _check(lib().qkv_pages_compact_workspace(pages, ctypes.byref(out)), "qkv_pages_compact_workspace")
    return out.value


def pages_compact(pages, status, live=None, workspace=None, stream=None):
    """Moves the pages in use to the front of the pool; live: device int32 [1] for their number, or None."""
    if workspace is None:
        workspace = _scratch(pages_compact_workspace(pages), pages.device, stream)
    lp = None if live is None else _of_pages(live, pages, torch.int32, (1,), "live")
    _check(lib().qkv_pages_compact(pages, lp, _of_pages(workspace, pages, torch.uint8, workspace.shape, "workspace"), workspace.numel(),
                                   _status_of_pages(status, pages), _here(pages, stream)), "qkv_pages_compact")


def _paged_query(pages, q, softmax_scale, out, out_type, lse, layer, window, sinks, workspace, status):
    shape, strides = q.shape, q.stride()
    if len(shape) != 3 or shape[2] != pages.head_dim or strides[2] != 1 or q.dtype is not pages.dtype or q.device != pages.device:
        raise ValueError("q must be [tokens, q_heads, head_dim] of the pages' type and device, rows contiguous")
    x = PagedQuery(q.data_ptr(), strides[0], strides[1], shape[0])
    x.out_dev = _of_pages(out, pages, out_type, shape, "out")
    if lse is not None:
        x.lse_dev = _of_pages(lse, pages, torch.float32, shape[:2], "lse")
    if workspace is not None:
        x.workspace_dev, x.workspace_bytes = _of_pages(workspace, pages, torch.uint8, workspace.shape, "workspace"), workspace.numel()
    if status is not None:
        x.status_dev = _status_of_pages(status, pages)
    x.layer, x.q_heads, x.window, x.sinks, x.softmax_scale = layer, shape[1], window, sinks, softmax_scale
    return x


def paged_attend_workspace(pages, q_heads):
    out = ctypes.c_uint64(0)
    _check(lib().qkv_paged_attend_workspace(pages, int(q_heads), ctypes.byref(out)), "qkv_paged_attend_workspace")
    return out.value


def paged_attend(pages, q, softmax_scale, out, lse=None, layer=0, window=0, sinks=0, prior=None, workspace=None, status=None, stream=None):
    """Attention of one new token of every row over its pages.  q: device [rows, q_heads, head_dim] of the pages' type (a view with contiguous
    rows is fine); out: device float32 of the same shape; lse: float32 [rows, q_heads]; prior: (out, lse) of attention over other tokens
    (card_attend's), which the result then covers too."""
    if workspace is None:
        workspace = _scratch(paged_attend_workspace(pages, q.shape[1]), pages.device, stream)
    x = _paged_query(pages, q, softmax_scale, out, torch.float32, lse, layer, window, sinks, workspace, status)
    if prior is not None:
        x.prior_out_dev = _of_pages(prior[0], pages, torch.float32, q.shape, "prior[0]")
        x.prior_lse_dev = _of_pages(prior[1], pages, torch.float32, q.shape[:2], "prior[1]")
    _check(lib().qkv_paged_attend(pages, x, _here(pages, stream)), "qkv_paged_attend")
    return out, lse


def paged_prompt_workspace(pages, q_heads, tokens):
    """Bytes that are enough for every batch of up to `tokens` tokens."""
    out = ctypes.c_uint64(0)
    _check(lib().qkv_paged_prompt_workspace(pages, int(q_heads), int(tokens), ctypes.byref(out)), "qkv_paged_prompt_workspace")
    return out.value


def paged_prompt(pages, q, starts, softmax_scale, out, lse=None, layer=0, window=0, sinks=0, workspace=None, status=None, stream=None):
    """Attention of the rows' last tokens, those of row i at q[starts[i]:starts[i + 1]], each over what stands up to its own place.
    q: device [tokens, q_heads, head_dim] of the pages' type; starts: device int32 [rows + 1]; out: of the pages' type; lse: float32 [tokens, q_heads]."""
    if workspace is None:
        workspace = _scratch(paged_prompt_workspace(pages, q.shape[1], q.shape[0]), pages.device, stream)
    x = _paged_query(pages, q, softmax_scale, out, pages.dtype, lse, layer, window, sinks, workspace, status)
    x.starts_dev = _of_pages(starts, pages, torch.int32, (pages.rows + 1,), "starts")
    _check(lib().qkv_paged_prompt(pages, x, _here(pages, stream)), "qkv_paged_prompt")
    return out, lse
