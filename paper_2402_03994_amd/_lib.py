"""ctypes declarations of the C ABI in include/sketch.h, include/sketch_hvp.h and include/sketch_train.h
(argument marshalling only)."""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsketch.so")

SK_FJL, SK_FFD, SK_AFFD, SK_AFJL, SK_QK, SK_QKH, SK_AFJLQ, SK_AFFDQ, SK_AFJLF = range(9)
SK_F32, SK_BF16 = 0, 1
SK_I32, SK_I64 = 0, 1
SK_ADAMW_F32, SK_ADAMW_8BIT = 0, 1
STATUS = {0: "SK_OK", -1: "SK_EINVAL", -2: "SK_EDTYPE", -3: "SK_ENOMEM", -4: "SK_EHIP", -5: "SK_EUNSUPPORTED"}
STREAMS = {"sign": 1, "gauss": 2, "index": 3, "ffdperm": 4, "pi1": 5, "pi2": 6, "qka": 7, "qkb": 8, "qh": 9,
           "hvp": 10}
EXPORTS = ("sketch_create", "sketch_apply", "sketch_apply_noalloc", "sketch_apply_T", "sketch_destroy", "sketch_query",
           "sketch_debug_stream", "sketch_profile", "sketch_profile_read", "sketch_last_error",
           "sketch_status_string", "sk_hvp_create", "sk_hvp_apply", "sk_hvp_destroy", "sketch_hvp",
           "sketch_arnoldi_work_floats", "sketch_arnoldi_step", "sketch_arnoldi", "sk_hvp_profile",
           "sk_hvp_profile_read", "sketch_id_search_work_floats", "sketch_id_search", "sketch_embed", "sketch_embed_grad",
           "sketch_embed_grad_work_bytes", "sketch_token_logp", "sketch_token_logp_grad", "sketch_policy_loss",
           "sketch_preference_work_bytes", "sketch_preference_loss", "sketch_linear_logp_work_bytes",
           "sketch_linear_logp", "sketch_linear_logp_grad_work_bytes", "sketch_linear_logp_grad",
           "sketch_dropout", "sketch_balance_work_bytes", "sketch_balance_loss", "sketch_adamw_create",
           "sketch_adamw_state_elems", "sketch_adamw_apply", "sketch_adamw_moments", "sketch_adamw_destroy")
HVP_PROF_CLASSES = ["hvp_dots", "hvp_combine", "arnoldi_orth"]
HVP_MAX_RANK = 32
PROF_CLASSES = ["afjl_fold", "afjl_tail", "fwht", "prolog", "affd_fold", "gather", "ffd", "qk", "other",
                "affd_rows", "qk_xb", "qh_first", "qh_second", "qh_t", "ffd_t", "ff_rows", "ff_res",
                "ff_small", "fjl_t"]


class IdResult(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int64), ("status", ctypes.c_int32), ("rounds", ctypes.c_int32),
                ("L0", ctypes.c_double)]


class LayerShape(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("qk_da", ctypes.c_int32),
                ("qk_db", ctypes.c_int32)]


class Info(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("n_layers", ctypes.c_int32), ("D", ctypes.c_int64),
                ("seed", ctypes.c_uint64), ("total_numel", ctypes.c_int64), ("total_padded", ctypes.c_int64),
                ("workspace_bytes", ctypes.c_int64), ("rng_version", ctypes.c_int32), ("device", ctypes.c_int32)]


class Logits(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("targets", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("vocab", ctypes.c_int64), ("ld", ctypes.c_int64), ("scale", ctypes.c_float),
                ("dtype", ctypes.c_int), ("index", ctypes.c_int), ("device", ctypes.c_int32)]


class Linear(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_void_p), ("weight", ctypes.c_void_p), ("targets", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("vocab", ctypes.c_int64), ("width", ctypes.c_int64),
                ("ld_hidden", ctypes.c_int64), ("ld_weight", ctypes.c_int64), ("scale", ctypes.c_float),
                ("dtype", ctypes.c_int), ("index", ctypes.c_int), ("device", ctypes.c_int32)]


class AdamWStep(ctypes.Structure):
    _fields_ = [("step", ctypes.c_int64), ("lr", ctypes.c_double), ("beta1", ctypes.c_double),
                ("beta2", ctypes.c_double), ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double),
                ("max_norm", ctypes.c_double), ("grad_scale", ctypes.c_void_p), ("norm", ctypes.c_void_p),
                ("m", ctypes.c_void_p), ("v", ctypes.c_void_p), ("m_exp", ctypes.c_void_p),
                ("v_exp", ctypes.c_void_p)]


_lib = None


def load() -> ctypes.CDLL:
    """Load libsketch.so; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2402_03994_amd.build` "
                           "(or __graft_entry__.build()); there is no non-HIP fallback")
    L = ctypes.CDLL(LIB_PATH)
    P, i32, i64, u32, u64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_uint64
    L.sketch_create.argtypes = [ctypes.c_int, ctypes.POINTER(LayerShape), i32, i64, u64, u32, i32,
                                ctypes.POINTER(P)]
    L.sketch_create.restype = ctypes.c_int
    L.sketch_apply.argtypes = [P, ctypes.POINTER(P), ctypes.c_int, i64, P, i32, i32, i32, P]
    L.sketch_apply.restype = ctypes.c_int
    L.sketch_apply_noalloc.argtypes = [P, ctypes.POINTER(P), ctypes.c_int, i64, P, i32, i32, i32, P]
    L.sketch_apply_noalloc.restype = ctypes.c_int
    L.sketch_apply_T.argtypes = [P, P, i64, ctypes.POINTER(P), ctypes.c_int, ctypes.POINTER(P), i32, i32, P]
    L.sketch_apply_T.restype = ctypes.c_int
    L.sketch_destroy.argtypes = [P]
    L.sketch_destroy.restype = None
    L.sketch_query.argtypes = [P, ctypes.POINTER(Info)]
    L.sketch_query.restype = ctypes.c_int
    L.sketch_debug_stream.argtypes = [P, i32, i32, u64, u64, u64, P]
    L.sketch_debug_stream.restype = ctypes.c_int
    L.sketch_profile.argtypes = [P, ctypes.c_uint32]
    L.sketch_profile.restype = ctypes.c_int
    L.sketch_profile_read.argtypes = [P, P, P, P]
    L.sketch_profile_read.restype = ctypes.c_int
    L.sketch_last_error.argtypes = []
    L.sketch_last_error.restype = ctypes.c_char_p
    L.sketch_status_string.argtypes = [ctypes.c_int]
    L.sketch_status_string.restype = ctypes.c_char_p
    f32 = ctypes.c_float
    L.sk_hvp_create.argtypes = [ctypes.POINTER(LayerShape), i32, i32, P, f32, u64, i64, i32, ctypes.POINTER(P)]
    L.sk_hvp_create.restype = ctypes.c_int
    L.sk_hvp_apply.argtypes = [P, ctypes.POINTER(P), i64, ctypes.POINTER(P), P]
    L.sk_hvp_apply.restype = ctypes.c_int
    L.sk_hvp_destroy.argtypes = [P]
    L.sk_hvp_destroy.restype = None
    L.sketch_hvp.argtypes = [P, P, P, i64, P, P]
    L.sketch_hvp.restype = ctypes.c_int
    L.sketch_arnoldi_work_floats.argtypes = [i64, i32]
    L.sketch_arnoldi_work_floats.restype = i64
    L.sketch_arnoldi_step.argtypes = [P, i64, i32, P, i32, P, P]
    L.sketch_arnoldi_step.restype = ctypes.c_int
    L.sketch_arnoldi.argtypes = [P, P, P, i32, P, P, P]
    L.sketch_arnoldi.restype = ctypes.c_int
    L.sk_hvp_profile.argtypes = [P, u32]
    L.sk_hvp_profile.restype = ctypes.c_int
    L.sk_hvp_profile_read.argtypes = [P, P, P, P]
    L.sk_hvp_profile_read.restype = ctypes.c_int
    L.sketch_id_search_work_floats.argtypes = [i64]
    L.sketch_id_search_work_floats.restype = i64
    L.sketch_id_search.argtypes = [P, P, ctypes.POINTER(P), i64, f32, f32, i32, i32, P, P, P,
                                   ctypes.POINTER(IdResult), P]
    L.sketch_id_search.restype = ctypes.c_int
    LP, SP, XP = ctypes.POINTER(Logits), ctypes.POINTER(AdamWStep), ctypes.POINTER(Linear)
    for name, restype, args in (
            ("sketch_embed", ctypes.c_int, [P, ctypes.c_int, i64, i64, i64, P, ctypes.c_int, i64, f32, P, ctypes.c_int,
                                            i32, P]),
            ("sketch_embed_grad_work_bytes", i64, [i64, i64, i64]),
            ("sketch_embed_grad", ctypes.c_int, [P, ctypes.c_int, i64, P, ctypes.c_int, i64, i64, i64, i64, f32, P,
                                                 ctypes.c_int, i32, P, i64, i32, P]),
            ("sketch_token_logp", ctypes.c_int, [LP, P, P, P]),
            ("sketch_token_logp_grad", ctypes.c_int, [LP, P, P, P, i64, P]),
            ("sketch_policy_loss", ctypes.c_int, [LP, P, P, P, P, f32, f32, f32, P, P, P, P, i64, P]),
            ("sketch_preference_work_bytes", i64, [i64]),
            ("sketch_preference_loss", ctypes.c_int, [LP, P, ctypes.c_int, i64, P, f32, f32, i32, P, P, P, P, i64, P,
                                                      i64, P]),
            ("sketch_linear_logp_work_bytes", i64, [XP]),
            ("sketch_linear_logp", ctypes.c_int, [XP, P, P, P, i64, P]),
            ("sketch_linear_logp_grad_work_bytes", i64, [XP, i64, i32, i32]),
            ("sketch_linear_logp_grad", ctypes.c_int, [XP, i64, P, P, P, i64, P, ctypes.c_int, i32, P, i64, P]),
            ("sketch_dropout", ctypes.c_int, [P, ctypes.c_int, i64, i64, i64, P, i64, P, i64, ctypes.c_double, u64, i64, P,
                                              i64, i32, P]),
            ("sketch_balance_work_bytes", i64, [i64]),
            ("sketch_balance_loss", ctypes.c_int, [P, ctypes.c_int, i64, i64, i64, P, ctypes.c_int, i64, f32, P, P, P, P,
                                                   i64, P, i64, i32, P]),
            ("sketch_adamw_create", ctypes.c_int, [P, P, i32, ctypes.c_int, u64, i32, ctypes.POINTER(P)]),
            ("sketch_adamw_state_elems", i64, [P]),
            ("sketch_adamw_apply", ctypes.c_int, [P, SP, ctypes.POINTER(P), ctypes.c_int, ctypes.POINTER(P),
                                                  ctypes.c_int, ctypes.POINTER(P), P]),
            ("sketch_adamw_moments", ctypes.c_int, [P, P, P, P, P, P, P, P]),
            ("sketch_adamw_destroy", None, [P])):
        fn = getattr(L, name)
        fn.argtypes, fn.restype = args, restype
    _lib = L
    return L


class SketchError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code


def check(rc: int) -> None:
    if rc != 0:
        raise SketchError(rc, load().sketch_last_error().decode())
