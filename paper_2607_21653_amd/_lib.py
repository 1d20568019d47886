"""ctypes binding of libmolt.so: argument marshalling only.

Every function takes torch tensors that already live on the GPU, checks dtypes,
shapes and contiguity, allocates outputs and the workspace with torch (device
memory is torch's job), and calls the C entry point of the same name on torch's
current stream. There is no fallback: if the library is missing or no GPU is
present, the call raises."""
import ctypes
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmolt.so")
CALLS_PATH = os.path.join(HERE, "_calls.so")

MOLT_F32, MOLT_BF16, MOLT_FP8_E4M3 = 0, 1, 2
MOLT_ERR_WORKSPACE = -3
MOLT_KV_MX = 0x100                # MOLT_KV_MX of include/molt.h
NOALLOC_SCRATCH_BYTES = 8 << 20   # MOLT_NOALLOC_SCRATCH_BYTES of include/molt.h
DTYPE_CODE = {torch.float32: MOLT_F32, torch.bfloat16: MOLT_BF16, torch.uint8: MOLT_FP8_E4M3}
NAME_CODE = {"f32": MOLT_F32, "bf16": MOLT_BF16, "fp8": MOLT_FP8_E4M3}

_lib = None
_calls = None                     # the module of csrc/binding/calls.cpp, from its first call on

c_int, c_size, c_vp, c_float = ctypes.c_int, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_float


class MoltModel(ctypes.Structure):
    _fields_ = [(n, c_int) for n in ("n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim",
                                     "n_experts", "top_k", "d_ff", "vocab")] + [
        ("rms_eps", c_float), ("rope_theta", c_float), ("dtype", c_int), ("expert_dtype", c_int),
        ("embed", c_vp), ("final_norm", c_vp), ("lm_head", c_vp),
        ("attn_norm", c_vp), ("w_qkv", c_vp), ("w_o", c_vp), ("moe_norm", c_vp),
        ("w_router", c_vp), ("router_bias", c_vp), ("w_gate_up", c_vp), ("w_down", c_vp),
        ("s_gate_up", c_vp), ("s_down", c_vp)]


class MoltKV(ctypes.Structure):
    _fields_ = [("k_cache", c_vp), ("v_cache", c_vp), ("block_tables", c_vp),
                ("context_lens", c_vp), ("max_blocks_per_seq", c_int), ("num_blocks", c_int),
                ("block_size", c_int)]


class MoltMtp(ctypes.Structure):
    _fields_ = [("enorm", c_vp), ("hnorm", c_vp), ("eh_proj", c_vp),
                ("layer", ctypes.POINTER(MoltModel))]


_SIGS = {
    "molt_last_error": (ctypes.c_char_p, []),
    "molt_version": (c_int, []),
    "molt_spec_accept_workspace_size": (c_size, [c_int, c_int, c_int]),
    "molt_spec_accept": (c_int, [c_vp, c_vp, c_vp, c_vp, c_int, c_int, c_int, c_vp, c_vp, c_vp,
                                 c_vp, c_size, c_vp]),
    "molt_spec_accept_noalloc": (c_int, [c_vp, c_vp, c_vp, c_vp, c_int, c_int, c_int, c_vp, c_vp,
                                         c_vp, c_vp]),
    "molt_moe_layer_workspace_size": (c_size, [c_int] * 5 + [c_int, c_int]),
    "molt_moe_layer": (c_int, [c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_int, c_int, c_int,
                               c_int, c_int, c_int, c_int, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp,
                               c_vp, c_vp, c_size, c_vp]),
    "molt_pack_weights": (c_int, [c_vp, c_vp, ctypes.c_longlong, ctypes.c_longlong, c_vp]),
    "molt_dense_gemm_workspace_size": (c_size, [c_int, c_int, c_int, c_int]),
    "molt_dense_gemm": (c_int, [c_vp, c_vp, c_vp, c_int, c_int, c_int, c_int, c_int, c_vp, c_size, c_vp]),
    "molt_paged_attention_workspace_size": (c_size, [c_int] * 6),
    "molt_paged_attention": (c_int, [c_vp, c_vp, c_vp, c_vp, c_vp, c_int, c_int, c_int, c_int,
                                     c_int, c_int, c_int, c_vp, c_vp, c_size, c_vp]),
    "molt_kvq_write": (c_int, [c_vp, c_vp, ctypes.c_longlong, ctypes.c_longlong, c_vp, c_vp, c_vp, c_vp,
                               c_vp, c_int, c_int, c_int, c_int, c_int, c_int, c_int, c_vp]),
    "molt_kvq_read": (c_int, [c_vp, c_vp, c_vp, c_vp, c_vp, c_int, c_int, c_int, c_int, c_int, c_int,
                              c_int, c_vp, c_vp, c_vp]),
    "molt_paged_attention_kvq_workspace_size": (c_size, [c_int] * 6),
    "molt_paged_attention_kvq": (c_int, [c_vp, c_vp, c_vp, c_vp, c_vp, c_int, c_int, c_int, c_int,
                                         c_int, c_int, c_int, c_int, c_vp, c_vp, c_size, c_vp]),
    "molt_kvq_workspace_extra": (c_size, [ctypes.POINTER(MoltModel), c_int, c_int, c_int]),
    "molt_plan_blocks_workspace_size": (c_size, [c_int, c_int]),
    "molt_plan_blocks": (c_int, [c_vp] * 6 + [c_int] * 4 + [c_vp, c_vp, c_vp, c_size, c_vp]),
    "molt_kv_write": (c_int, [c_vp, c_vp, ctypes.c_longlong, ctypes.c_longlong, c_vp, c_int, c_int, c_int, c_int,
                              c_int, c_vp, c_vp, c_vp]),
    "molt_key_bounds_update": (c_int, [c_vp] * 5 + [c_int] * 7 + [c_vp]),
    "molt_key_bounds_read": (c_int, [c_vp, c_vp, c_int, c_int, c_int, c_int, c_vp, c_vp, c_vp]),
    "molt_select_blocks_workspace_size": (c_size, [c_int] * 6),
    "molt_select_blocks": (c_int, [c_vp] * 5 + [c_int] * 11 + [c_vp, c_vp, c_size, c_vp]),
    "molt_paged_attention_blocks_workspace_size": (c_size, [c_int] * 6),
    "molt_paged_attention_blocks": (c_int, [c_vp] * 6 + [c_int] * 9 + [c_vp, c_vp, c_size, c_vp]),
    "molt_decoder_workspace_size": (c_size, [ctypes.POINTER(MoltModel), c_int, c_int, c_int]),
    "molt_decoder_forward": (c_int, [ctypes.POINTER(MoltModel), ctypes.POINTER(MoltKV), c_int,
                                     c_int, c_vp, c_vp, c_vp, c_size, c_vp]),
    "molt_profile_enable": (c_int, [c_int]),
    "molt_profile_every": (c_int, [c_int]),
    "molt_profile_read": (c_int, [c_int, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(c_int)]),
    "molt_verify_step_workspace_size": (c_size, [ctypes.POINTER(MoltModel), c_int, c_int, c_int]),
    "molt_verify_step": (c_int, [ctypes.POINTER(MoltModel), ctypes.POINTER(MoltKV), c_int, c_int,
                                 c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp,
                                 c_size, c_vp]),
    "molt_prefill_workspace_size": (c_size, [ctypes.POINTER(MoltModel), c_int, c_int, c_int]),
    "molt_prefill": (c_int, [ctypes.POINTER(MoltModel), ctypes.POINTER(MoltKV), c_int, c_int, c_vp,
                             c_vp, c_vp, c_vp, c_vp, c_vp, c_size, c_vp]),
    "molt_prefix_cache_create": (c_vp, [c_int]),
    "molt_prefix_cache_destroy": (None, [c_vp]),
    "molt_prefix_cache_acquire": (c_int, [c_vp, c_vp, c_int, c_int, c_vp, c_int,
                                          ctypes.POINTER(c_int)]),
    "molt_prefix_cache_commit": (c_int, [c_vp, c_vp, c_int, c_vp, c_int]),
    "molt_prefix_cache_release": (c_int, [c_vp, c_vp, c_int]),
    "molt_prefix_cache_stats": (c_int, [c_vp, ctypes.POINTER(ctypes.c_longlong)]),
    "molt_score_tokens_workspace_size": (c_size, [ctypes.POINTER(MoltModel), c_int, c_int, c_int]),
    "molt_score_tokens": (c_int, [ctypes.POINTER(MoltModel), ctypes.POINTER(MoltKV), c_int, c_int,
                                  c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_size, c_vp]),
    "molt_mtp_draft_workspace_size": (c_size, [ctypes.POINTER(MoltModel), ctypes.POINTER(MoltMtp),
                                               c_int, c_int, c_int]),
    "molt_mtp_draft_window_workspace_size": (c_size, [ctypes.POINTER(MoltModel), ctypes.POINTER(MoltMtp),
                                                      c_int, c_int, c_int, c_int]),
    "molt_mtp_draft_window": (c_int, [ctypes.POINTER(MoltModel), ctypes.POINTER(MoltMtp),
                                      ctypes.POINTER(MoltKV), c_int, c_int, c_int, c_vp, c_vp, c_vp,
                                      c_vp, c_vp, c_vp, c_vp, c_vp, c_size, c_vp]),
    "molt_mtp_draft": (c_int, [ctypes.POINTER(MoltModel), ctypes.POINTER(MoltMtp),
                               ctypes.POINTER(MoltKV), c_int, c_int, c_vp, c_vp, c_vp, c_vp, c_vp,
                               c_vp, c_vp, c_vp, c_size, c_vp]),
}


class MoltError(RuntimeError):
    pass


def load(path=LIB_PATH):
    """Loads the library (once). Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise MoltError(f"{path} is missing: build it with `python -m paper_2607_21653_amd.build`")
    lib = ctypes.CDLL(path)
    for name, (res, args) in _SIGS.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _load_calls():
    """The module of csrc/binding/calls.cpp, which the calls of sparse attention go through and no others need."""
    global _calls
    if _calls is None:
        lib = load()
        if not os.path.exists(CALLS_PATH):
            raise MoltError(f"{CALLS_PATH} is missing: build it with `python -m paper_2607_21653_amd.build`")
        try:
            from . import _calls as calls
        except ImportError as e:
            raise MoltError(f"{CALLS_PATH} cannot be loaded, build it for this torch with "
                            f"`python -m paper_2607_21653_amd.build`: {e}") from e
        calls.set_entries(MoltError, *(ctypes.cast(getattr(lib, "molt_" + name), c_vp).value for name in (
            "last_error", "plan_blocks", "plan_blocks_workspace_size", "kv_write", "key_bounds_update", "key_bounds_read",
            "select_blocks", "select_blocks_workspace_size", "paged_attention_blocks", "paged_attention_blocks_workspace_size",
            "plan_blocks_takes", "key_bounds_read_takes", "select_blocks_takes", "paged_attention_blocks_takes")))
        _calls = calls
    return _calls


def exported_symbols():
    return list(_SIGS)


def _check(status, name):
    if status != 0:
        msg = _lib.molt_last_error().decode()
        raise MoltError(f"{name} returned {status}: {msg}")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _dev(t, dtype, shape=None, name="tensor"):
    if t is None:
        return None
    if not t.is_cuda:
        raise MoltError(f"{name} must be a GPU tensor")
    if dtype is not None and t.dtype != dtype:
        raise MoltError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if not t.is_contiguous():
        raise MoltError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise MoltError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _workspace(nbytes, device, ws=None):
    if nbytes == 0:
        return None, 0
    if ws is not None and ws.numel() >= nbytes:
        return ws, ws.numel()
    t = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return t, nbytes


def _call(name, call, nbytes, device, ws):
    """call(workspace address, its bytes) with the caller's workspace, also a smaller one where the
    library takes it (coarser attention splits), else with one of nbytes."""
    have = 0 if ws is None else ws.numel()
    if have:
        status = call(_ptr(ws), have)
        if have >= nbytes or status != MOLT_ERR_WORKSPACE:
            return _check(status, name)
    t, nb = _workspace(nbytes, device)
    _check(call(_ptr(t), nb), name)


# ------------------------------------------------------------------ spec accept

def spec_accept(logits, draft_tokens, uniforms, draft_probs=None, out=None, workspace=None):
    """logits [B, k+1, V] f32; draft_tokens [B, k] i32; uniforms [B, k+1] f32;
    draft_probs [B, k, V] f32 or None (one-hot q). Returns (tokens, n_accepted, logprobs)."""
    lib = load()
    B, kp1, V = logits.shape
    k = kp1 - 1
    _dev(logits, torch.float32, name="logits")
    _dev(uniforms, torch.float32, (B, kp1), "uniforms")
    if k > 0:
        _dev(draft_tokens, torch.int32, (B, k), "draft_tokens")
    _dev(draft_probs, torch.float32, (B, k, V), "draft_probs")
    dev = logits.device
    if out is None:
        out = (torch.empty(B, kp1, dtype=torch.int32, device=dev),
               torch.empty(B, dtype=torch.int32, device=dev),
               torch.empty(B, kp1, dtype=torch.float32, device=dev))
    toks, n, lp = out
    ws, nb = _workspace(lib.molt_spec_accept_workspace_size(B, k, V), dev, workspace)
    st = lib.molt_spec_accept(_ptr(logits), _ptr(draft_probs), _ptr(draft_tokens) if k > 0 else None,
                              _ptr(uniforms), B, k, V, _ptr(toks), _ptr(n), _ptr(lp), _ptr(ws), nb,
                              _stream())
    _check(st, "molt_spec_accept")
    return toks, n, lp


def spec_accept_noalloc(logits, draft_tokens, uniforms, draft_probs=None, out=None):
    """molt_spec_accept_noalloc: spec_accept with the library's fixed per-GPU scratch array
    instead of a workspace (no device allocation inside the call when `out` is given)."""
    lib = load()
    B, kp1, V = logits.shape
    k = kp1 - 1
    _dev(logits, torch.float32, name="logits")
    _dev(uniforms, torch.float32, (B, kp1), "uniforms")
    if k > 0:
        _dev(draft_tokens, torch.int32, (B, k), "draft_tokens")
    _dev(draft_probs, torch.float32, (B, k, V), "draft_probs")
    dev = logits.device
    if out is None:
        out = (torch.empty(B, kp1, dtype=torch.int32, device=dev),
               torch.empty(B, dtype=torch.int32, device=dev),
               torch.empty(B, kp1, dtype=torch.float32, device=dev))
    toks, n, lp = out
    st = lib.molt_spec_accept_noalloc(_ptr(logits), _ptr(draft_probs),
                                      _ptr(draft_tokens) if k > 0 else None, _ptr(uniforms), B, k, V,
                                      _ptr(toks), _ptr(n), _ptr(lp), _stream())
    _check(st, "molt_spec_accept_noalloc")
    return toks, n, lp


# ------------------------------------------------------------------ weight layout

def pack_weights(w):
    """w (row-major, last dim contiguous) in the library's tiled GEMM operand layout
    (molt_pack_weights). Same dtype; shape [R, last] with the rows padded to a multiple
    of 32, except that a matrix whose row count is already such a multiple keeps its shape."""
    lib = load()
    _dev(w, None, name="w")
    rows = w.numel() // w.shape[-1]
    padded = (rows + 31) // 32 * 32
    shape = tuple(w.shape) if padded == rows else (padded, w.shape[-1])
    out = torch.empty(shape, dtype=w.dtype, device=w.device)
    _check(lib.molt_pack_weights(_ptr(w), _ptr(out), rows, w.shape[-1] * w.element_size(), _stream()),
           "molt_pack_weights")
    return out


def _rows(t):
    return t.numel() // t.shape[-1]


# ------------------------------------------------------------------ MoE layer

def moe_layer(x, w_router, w_gate_up, w_down, top_k, router_bias=None, s_gate_up=None,
              s_down=None, replay_ids=None, want_routing=False, workspace=None, packed=False,
              n_experts=None):
    """x [T, d] (f32|bf16); weights as in molt.h (fp8 experts as uint8 codes): router and
    expert weights row-major (packed here, per call), or already tiled with packed=True
    (then give n_experts when the router's row count is not a multiple of 32).
    Returns out [T, d] f32, or (out, ids, weights, counts, offsets, perm) with want_routing."""
    lib = load()
    T, d = x.shape
    E = n_experts if n_experts is not None else w_router.shape[0]
    if not packed:
        _dev(w_router, x.dtype, (E, d), "w_router")
        w_router = pack_weights(w_router)
        w_gate_up, w_down = pack_weights(w_gate_up), pack_weights(w_down)
    F = w_gate_up.shape[1] // 2
    act = DTYPE_CODE[x.dtype]
    wdt = DTYPE_CODE[w_gate_up.dtype]
    _dev(x, None, name="x")
    _dev(w_router, x.dtype, ((E + 31) // 32 * 32 if E % 32 else E, d), "w_router")
    _dev(w_gate_up, None, (E, 2 * F, d), "w_gate_up")
    _dev(w_down, w_gate_up.dtype, (E, d, F), "w_down")
    _dev(router_bias, torch.float32, (E,), "router_bias")
    _dev(s_gate_up, torch.float32, (E, 2 * F), "s_gate_up")
    _dev(s_down, torch.float32, (E, d), "s_down")
    _dev(replay_ids, torch.int32, (T, top_k), "replay_ids")
    dev = x.device
    out = torch.empty(T, d, dtype=torch.float32, device=dev)
    ids = wts = counts = offsets = perm = None
    if want_routing:
        ids = torch.empty(T, top_k, dtype=torch.int32, device=dev)
        wts = torch.empty(T, top_k, dtype=torch.float32, device=dev)
        counts = torch.empty(E, dtype=torch.int32, device=dev)
        offsets = torch.empty(E + 1, dtype=torch.int32, device=dev)
        perm = torch.empty(T * top_k, dtype=torch.int32, device=dev)
    ws, nb = _workspace(lib.molt_moe_layer_workspace_size(T, d, E, top_k, F, act, wdt), dev, workspace)
    st = lib.molt_moe_layer(_ptr(x), _ptr(w_router), _ptr(router_bias), _ptr(w_gate_up), _ptr(w_down),
                            _ptr(s_gate_up), _ptr(s_down), T, d, E, top_k, F, act, wdt,
                            _ptr(replay_ids), _ptr(out), _ptr(ids), _ptr(wts), _ptr(counts),
                            _ptr(offsets), _ptr(perm), _ptr(ws), nb, _stream())
    _check(st, "molt_moe_layer")
    if want_routing:
        return out, ids, wts, counts, offsets, perm
    return out


# ------------------------------------------------------------------ dense GEMM

def dense_gemm(A, B, C=None, accumulate=False, workspace=None):
    """C [M, N] f32 = A [M, K] @ B [N, K]^T (+ C when accumulate); A, B f32 or bf16,
    row-major (packed into the tiled operand layout here)."""
    lib = load()
    M, K = A.shape
    N = B.shape[0]
    _dev(A, None, name="A")
    _dev(B, A.dtype, (N, K), "B")
    if C is None:
        C = torch.zeros(M, N, dtype=torch.float32, device=A.device)
    _dev(C, torch.float32, (M, N), "C")
    At, Bt = pack_weights(A), pack_weights(B)
    dt = DTYPE_CODE[A.dtype]
    ws, nb = _workspace(lib.molt_dense_gemm_workspace_size(M, N, K, dt), A.device, workspace)
    _check(lib.molt_dense_gemm(_ptr(At), _ptr(Bt), _ptr(C), M, N, K, dt, 1 if accumulate else 0,
                               _ptr(ws), nb, _stream()), "molt_dense_gemm")
    return C


# ------------------------------------------------------------------ paged attention

def paged_attention(q, k_cache, v_cache, block_tables, context_lens, k, workspace=None):
    """q [B*(1+k), Hq, D]; caches [nb, Hkv, 16, D] / [nb, Hkv, D, 16]; returns [T, Hq*D]."""
    lib = load()
    T, Hq, D = q.shape
    B = context_lens.shape[0]
    Hkv = k_cache.shape[1]
    if T != B * (k + 1):
        raise MoltError(f"q has {T} rows, expected B*(1+k) = {B * (k + 1)}")
    _dev(q, None, name="q")
    _dev(k_cache, q.dtype, name="k_cache")
    _dev(v_cache, q.dtype, name="v_cache")
    _dev(block_tables, torch.int32, name="block_tables")
    _dev(context_lens, torch.int32, (B,), "context_lens")
    maxb = block_tables.shape[1]
    out = torch.empty(T, Hq * D, dtype=q.dtype, device=q.device)

    def call(ws, nb):
        return lib.molt_paged_attention(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_tables),
                                        _ptr(context_lens), B, k, Hq, Hkv, D, maxb, DTYPE_CODE[q.dtype],
                                        _ptr(out), ws, nb, _stream())

    _call("molt_paged_attention", call, lib.molt_paged_attention_workspace_size(B, k, Hq, Hkv, D, maxb),
          q.device, workspace)
    return out


# ------------------------------------------------------------------ 4-bit KV cache

def kvq_cache(num_blocks, n_kv_heads, head_dim, device="cuda"):
    """Empty (k_cache, v_cache) of the 4-bit format (molt.h): uint8 [num_blocks, n_kv_heads, 17 D / 2]."""
    shape = (num_blocks, n_kv_heads, 17 * head_dim // 2)
    return (torch.zeros(shape, dtype=torch.uint8, device=device),
            torch.zeros(shape, dtype=torch.uint8, device=device))


# The calls below take 3 to 8 us on the GPU where they are small, and as long on the host: they ask each tensor
# for what they need once, and take the paths with messages only where something is wrong.
# (torch's own names for these two are not public, and missing where torch is built without GPU support, where the
# package's host parts work all the same)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
# of a device index, without a torch.cuda.Stream around it (2.6 us)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _kvq_caches(k_cache, v_cache, block_tables, starts):
    """Checks of a pair of caches and the tables; returns (device index, B, num_blocks, n_kv_heads, head_dim,
    max_blocks)."""
    dev = k_cache.get_device()
    shape, table = k_cache.shape, block_tables.shape
    if not (dev >= 0 and len(shape) == 3 and len(table) == 2 and v_cache.shape == shape
            and starts.dim() == 1 and starts.numel() == table[0]
            and k_cache.dtype is v_cache.dtype is torch.uint8 and block_tables.dtype is starts.dtype is torch.int32
            and v_cache.get_device() == block_tables.get_device() == starts.get_device() == dev
            and k_cache.is_contiguous() and v_cache.is_contiguous() and block_tables.is_contiguous()
            and starts.is_contiguous()) or shape[2] * 2 % 17:
        _dev(k_cache, torch.uint8, name="k_cache")
        if len(shape) != 3 or shape[2] * 2 % 17:
            raise MoltError(f"k_cache has shape {tuple(shape)}, expected [num_blocks, n_kv_heads, 17 * head_dim / 2]")
        _dev(v_cache, torch.uint8, shape, "v_cache")
        _dev(starts, torch.int32, (starts.numel(),), "context_lens")
        _dev(block_tables, torch.int32, name="block_tables")
        if len(table) != 2 or table[0] != starts.shape[0]:
            raise MoltError(f"block_tables has shape {tuple(table)}, expected ({starts.shape[0]}, max_blocks)")
        raise MoltError("k_cache, v_cache, block_tables and context_lens must be on one device")
    if dev != _current_device():
        raise MoltError(f"the caches are on device {dev}, the current device is {_current_device()}")
    return dev, table[0], shape[0], shape[1], shape[2] * 2 // 17, table[1]


def _same_device(t, dev, name):
    if t.get_device() != dev:
        raise MoltError(f"{name} must be a GPU tensor on device {dev}, the caches', is on {t.device}")


def _kvq_lens(lens, B, dev):
    """Address of lens, or None."""
    if lens is None:
        return None
    _dev(lens, torch.int32, (B,), "lens")
    _same_device(lens, dev, "lens")
    return lens.data_ptr()


def _rows_stride(t, dtype, T, H, D, dev, name):
    """Row stride (elements) of rows [T, H, D] whose heads are contiguous, e.g. a slice of fused QKV rows."""
    if t.dtype is not dtype:
        raise MoltError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.shape != (T, H, D):
        raise MoltError(f"{name} has shape {tuple(t.shape)}, expected {(T, H, D)}")
    row, head, dim = t.stride()
    if dim != 1 or (H > 1 and head != D) or (T > 1 and row < H * D):
        raise MoltError(f"{name} must have contiguous heads in rows that do not overlap, strides are {t.stride()}")
    _same_device(t, dev, name)
    return row if T > 1 else H * D


def kvq_write(k, v, k_cache, v_cache, block_tables, context_lens, n, lens=None):
    """Writes rows k, v [B*n, Hkv, D] (f32|bf16; row-strided views will do) into the 4-bit cache at
    positions context_lens[b] + j, j < n (j < lens[b] if given)."""
    lib = _lib or load()
    dev, B, nb, Hkv, D, maxb = _kvq_caches(k_cache, v_cache, block_tables, context_lens)
    dt = k.dtype
    if dt is not torch.bfloat16 and dt is not torch.float32:
        raise MoltError(f"k has dtype {dt}, expected float32 or bfloat16")
    ks, vs = _rows_stride(k, dt, B * n, Hkv, D, dev, "k"), _rows_stride(v, dt, B * n, Hkv, D, dev, "v")
    status = lib.molt_kvq_write(k.data_ptr(), v.data_ptr(), ks, vs, k_cache.data_ptr(), v_cache.data_ptr(),
                                block_tables.data_ptr(), context_lens.data_ptr(), _kvq_lens(lens, B, dev), B, n,
                                Hkv, D, maxb, nb, DTYPE_CODE[dt], _raw_stream(dev))
    if status:
        _check(status, "molt_kvq_write")


def kvq_read(k_cache, v_cache, block_tables, starts, n, lens=None, dtype=torch.bfloat16):
    """Positions starts[b] + j, j < n, of the 4-bit cache as (k, v) [B*n, Hkv, D] of dtype (bf16|f32); rows
    j >= lens[b], and rows without a place in the table, are zeros."""
    lib = _lib or load()
    dev, B, nb, Hkv, D, maxb = _kvq_caches(k_cache, v_cache, block_tables, starts)
    if dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise MoltError(f"dtype is {dtype}, expected float32 or bfloat16")
    if n < 1:
        raise MoltError(f"n = {n} must be >= 1")
    lens = _kvq_lens(lens, B, dev)
    k = torch.empty(B * n, Hkv, D, dtype=dtype, device=k_cache.device)
    v = torch.empty_like(k)
    status = lib.molt_kvq_read(k_cache.data_ptr(), v_cache.data_ptr(), block_tables.data_ptr(), starts.data_ptr(),
                               lens, B, n, Hkv, D, maxb, nb, DTYPE_CODE[dtype], k.data_ptr(), v.data_ptr(),
                               _raw_stream(dev))
    if status:
        _check(status, "molt_kvq_read")
    return k, v


def paged_attention_kvq_workspace_size(B, k, n_q_heads, n_kv_heads, head_dim, max_blocks):
    return load().molt_paged_attention_kvq_workspace_size(B, k, n_q_heads, n_kv_heads, head_dim, max_blocks)


def paged_attention_kvq(q, k_cache, v_cache, block_tables, context_lens, k, workspace=None):
    """paged_attention over a 4-bit cache: q [B*(1+k), Hq, D] (f32|bf16); returns [T, Hq*D] of q's dtype."""
    lib = _lib or load()
    dev, B, nb, Hkv, D, maxb = _kvq_caches(k_cache, v_cache, block_tables, context_lens)
    dt, shape = q.dtype, q.shape
    if dt is not torch.bfloat16 and dt is not torch.float32:
        raise MoltError(f"q has dtype {dt}, expected float32 or bfloat16")
    if len(shape) != 3:
        raise MoltError(f"q has shape {tuple(shape)}, expected [B*(1+k), Hq, D]")
    T, Hq, _ = shape
    if T != B * (k + 1) or shape[2] != D or not q.is_contiguous():
        _dev(q, None, (B * (k + 1), Hq, D), "q")
    _same_device(q, dev, "q")
    ws, have = None, 0
    if workspace is not None:
        _same_device(workspace, dev, "workspace")
        if not workspace.is_contiguous():
            raise MoltError("workspace must be contiguous")
        ws, have = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    out = q.new_empty(T, Hq * D)
    args = (q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), block_tables.data_ptr(), context_lens.data_ptr(),
            B, k, Hq, Hkv, D, maxb, nb, DTYPE_CODE[dt], out.data_ptr())
    status = lib.molt_paged_attention_kvq(*args, ws, have, _raw_stream(dev))
    if status == MOLT_ERR_WORKSPACE:     # none, or one that is too small
        own, have = _workspace(lib.molt_paged_attention_kvq_workspace_size(B, k, Hq, Hkv, D, maxb), q.device)
        status = lib.molt_paged_attention_kvq(*args, _ptr(own), have, _raw_stream(dev))
    if status:
        _check(status, "molt_paged_attention_kvq")
    return out


# ------------------------------------------------------------------ sparse attention over listed blocks

# The calls below take 3 to 8 us on the GPU where they are small. They go through _calls, which looks their arguments over
# in C++ and returns None where it does not take them: then the reason is found here, argument by argument.

def _here(t, name):
    """Index of a tensor's device, which must be the current one."""
    if not isinstance(t, torch.Tensor):
        raise MoltError(f"{name} must be a GPU tensor, is {type(t).__name__}")
    dev = t.get_device()
    if dev < 0:
        raise MoltError(f"{name} must be a GPU tensor")
    if dev != _current_device():
        raise MoltError(f"{name} is on device {dev}, the current device is {_current_device()}")
    return dev


def _kinds(tensors, optional=None, **numbers):
    """Refuses the first of a call's arguments (by name) that is no tensor, or no whole number from its least value,
    (value, least), to 2^31 - 1. Optional tensors may be None."""
    for name, t in tensors.items():
        if not isinstance(t, torch.Tensor):
            raise MoltError(f"{name} must be a GPU tensor, is {type(t).__name__}")
    for name, t in (optional or {}).items():
        if t is not None and not isinstance(t, torch.Tensor):
            raise MoltError(f"{name} must be a GPU tensor or None, is {type(t).__name__}")
    for name, (value, least) in numbers.items():
        if isinstance(value, torch.Tensor) or not hasattr(value, "__index__"):
            raise MoltError(f"{name} = {value!r} must be a whole number")
        if not least <= value:
            raise MoltError(f"{name} = {value} must be >= {least}")
        if value > 0x7fffffff:
            raise MoltError(f"{name} = {value} must be < 2^31")


def _fits(name, t, dtype, shape, dev):
    """Refuses a tensor that is not of dtype (float: bf16 or f32; None: any) and shape (None: any, also of one of its
    sizes), contiguous and on device dev; returns its shape. None is passed over."""
    if t is None:
        return None
    if shape is not None and (len(shape) != t.dim() or any(w is not None and w != n for w, n in zip(shape, t.shape))):
        raise MoltError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if dtype is float:
        dtype = t.dtype
        if dtype is not torch.bfloat16 and dtype is not torch.float32:
            raise MoltError(f"{name} has dtype {dtype}, expected float32 or bfloat16")
    _dev(t, dtype, None, name)
    _same_device(t, dev, name)
    return t.shape


def _fits_caches(k_cache, v_cache, dev):
    """(num_blocks, n_kv_heads, head_dim) of a cache"""
    nb, H, _, D = _fits("k_cache", k_cache, float, (None, None, 16, None), dev)
    _fits("v_cache", v_cache, k_cache.dtype, (nb, H, D, 16), dev)
    return nb, H, D


def _fits_bounds(bounds, dev):
    """(num_blocks, n_kv_heads, head_dim) of the bounds of a cache's keys"""
    nb, H, size = _fits("bounds", bounds, torch.uint8, (None, None, None), dev)
    if size <= 16 or size % 2:
        raise MoltError(f"bounds has shape {tuple(bounds.shape)}, expected (num_blocks, n_kv_heads, 2 * head_dim + 16)")
    return nb, H, (size - 16) // 2


def _fits_table(block_tables, dev, **rows):
    """The number of sequences, of a table and int32 tensors of one number each"""
    B, _ = _fits("block_tables", block_tables, torch.int32, (None, None), dev)
    for name, t in rows.items():
        _fits(name, t, torch.int32, (B,), dev)
    return B


def _not_taken(call):
    raise MoltError(f"{call}: a size among its tensors' is too large")


def block_pool(num_blocks, device="cuda"):
    """A pool for plan_blocks in which blocks 0 .. num_blocks - 1 are free: int32 [2 + num_blocks]."""
    pool = torch.arange(-2, num_blocks, dtype=torch.int32, device=device)
    pool[0], pool[1] = 0, num_blocks
    return pool


def plan_blocks(block_tables, n_blocks, context_lens, n_new, pool, n, n_shared=None):
    """Lets the block tables follow the lengths (molt_plan_blocks), all on the GPU and in place: sequence b gets the
    blocks that rows context_lens[b] .. + n_new[b] - 1 need from pool, or gives its own back where n_new[b] < 0.
    Returns (slots [B*n] i32 for kv_write, -1 where there is no row; placed [B] i32, rows that have slots)."""
    calls = _calls or _load_calls()
    dev = _here(block_tables, "block_tables")
    done = calls.plan(block_tables, n_blocks, context_lens, n_new, pool, n, n_shared, dev, _raw_stream(dev))
    if done is None:
        _kinds(dict(block_tables=block_tables, n_blocks=n_blocks, context_lens=context_lens, n_new=n_new, pool=pool),
               dict(n_shared=n_shared), n=(n, 1))
        _fits_table(block_tables, dev, n_blocks=n_blocks, context_lens=context_lens, n_new=n_new, n_shared=n_shared)
        if _fits("pool", pool, torch.int32, (None,), dev)[0] < 3:
            raise MoltError(f"pool has shape {tuple(pool.shape)}, expected (2 + num_blocks,)")
        _not_taken("molt_plan_blocks")
    return done


def kv_write(k, v, k_cache, v_cache, slots):
    """Writes rows k, v [T, Hkv, D] (row-strided views will do) into a bf16 or f32 cache at slots [T] i32 (block * 16 +
    token, as plan_blocks gives them); rows whose slot is outside the cache are left out."""
    calls = _calls or _load_calls()
    dev = _here(k_cache, "k_cache")
    if calls.write(k, v, k_cache, v_cache, slots, dev, _raw_stream(dev)) is None:
        _kinds(dict(k=k, v=v, k_cache=k_cache, v_cache=v_cache, slots=slots))
        _, H, D = _fits_caches(k_cache, v_cache, dev)
        T, = _fits("slots", slots, torch.int32, (None,), dev)
        for name, t in (("k", k), ("v", v)):
            if t.get_device() < 0:
                raise MoltError(f"{name} must be a GPU tensor")
            _rows_stride(t, k_cache.dtype, T, H, D, dev, name)
        _not_taken("molt_kv_write")


def key_bounds(num_blocks, n_kv_heads, head_dim, device="cuda"):
    """Empty bounds of a cache's keys (molt.h): uint8 [num_blocks, n_kv_heads, 2 D + 16]."""
    return torch.zeros(num_blocks, n_kv_heads, 2 * head_dim + 16, dtype=torch.uint8, device=device)


def key_bounds_update(k_cache, bounds, block_tables, starts, n, lens=None):
    """Bounds of the keys of the blocks that hold positions starts[b] + j, j < n (j < lens[b] if given), after
    kv_write of these rows."""
    calls = _calls or _load_calls()
    dev = _here(k_cache, "k_cache")
    if calls.update(k_cache, bounds, block_tables, starts, n, lens, dev, _raw_stream(dev)) is None:
        _kinds(dict(k_cache=k_cache, bounds=bounds, block_tables=block_tables, starts=starts), dict(lens=lens), n=(n, 1))
        nb, H, _, D = _fits("k_cache", k_cache, float, (None, None, 16, None), dev)
        _fits("bounds", bounds, torch.uint8, (nb, H, 2 * D + 16), dev)
        _fits_table(block_tables, dev, starts=starts, lens=lens)
        _not_taken("molt_key_bounds_update")


def key_bounds_read(bounds, ids):
    """The bounds of blocks ids [M] i32 of the cache as values: (largest, smallest) f32 [M, Hkv, D]."""
    calls = _calls or _load_calls()
    dev = _here(bounds, "bounds")
    done = calls.read(bounds, ids, dev, _raw_stream(dev))
    if done is None:
        _kinds(dict(bounds=bounds, ids=ids))
        _fits_bounds(bounds, dev)
        if _fits("ids", ids, torch.int32, (None,), dev)[0] < 1:
            raise MoltError("ids is empty")
        _not_taken("molt_key_bounds_read")
    return done


def select_blocks_workspace_size(B, k, n_q_heads, n_kv_heads, head_dim, max_blocks):
    return load().molt_select_blocks_workspace_size(B, k, n_q_heads, n_kv_heads, head_dim, max_blocks)


def select_blocks(q, bounds, block_tables, context_lens, k, n_select, n_first=1, n_last=2, lens=None, workspace=None):
    """For each query position (q [B*(1+k), Hq, D], f32|bf16, at context_lens[b] + j) and kv head the n_select blocks
    of largest score by the keys' bounds (molt_select_blocks), the first n_first and last n_last among them: i32
    [B*(1+k), Hkv, n_select], ascending, then -1. Rows j >= lens[b] have empty lists."""
    calls = _calls or _load_calls()
    dev = _here(bounds, "bounds")
    done = calls.select(q, bounds, block_tables, context_lens, k, n_select, n_first, n_last, lens, workspace, dev,
                        _raw_stream(dev))
    if done is None:
        _kinds(dict(q=q, bounds=bounds, block_tables=block_tables, context_lens=context_lens),
               dict(lens=lens, workspace=workspace), k=(k, 0), n_select=(n_select, 1), n_first=(n_first, 0),
               n_last=(n_last, 1))
        _, _, D = _fits_bounds(bounds, dev)
        B = _fits_table(block_tables, dev, context_lens=context_lens, lens=lens)
        _fits("q", q, float, (B * (int(k) + 1), None, D), dev)
        _fits("workspace", workspace, None, None, dev)
        _not_taken("molt_select_blocks")
    return done


def paged_attention_blocks_workspace_size(B, k, n_q_heads, n_kv_heads, head_dim, n_list):
    return load().molt_paged_attention_blocks_workspace_size(B, k, n_q_heads, n_kv_heads, head_dim, n_list)


def paged_attention_blocks(q, k_cache, v_cache, block_tables, context_lens, k, blocks, workspace=None):
    """paged_attention over the blocks that blocks [B*(1+k), Hkv, N] i32 lists for each position and kv head
    (select_blocks; -1: none): returns [B*(1+k), Hq*D] of q's dtype."""
    calls = _calls or _load_calls()
    dev = _here(k_cache, "k_cache")
    done = calls.attend(q, k_cache, v_cache, block_tables, context_lens, k, blocks, workspace, dev, _raw_stream(dev))
    if done is None:
        _kinds(dict(q=q, k_cache=k_cache, v_cache=v_cache, block_tables=block_tables, context_lens=context_lens,
                    blocks=blocks), dict(workspace=workspace), k=(k, 0))
        _, H, D = _fits_caches(k_cache, v_cache, dev)
        B = _fits_table(block_tables, dev, context_lens=context_lens)
        _fits("q", q, k_cache.dtype, (B * (int(k) + 1), None, D), dev)
        _fits("blocks", blocks, torch.int32, (B * (int(k) + 1), H, None), dev)
        _fits("workspace", workspace, None, None, dev)
        _not_taken("molt_paged_attention_blocks")
    return done


# ------------------------------------------------------------------ model / decoder / step

class Model:
    """Holds the device weights of a decoder and the molt_model struct that points at them.
    layers: list of dicts with attn_norm, w_qkv, w_o, moe_norm, w_router, w_gate_up, w_down,
    optional router_bias, s_gate_up, s_down. head: dict with embed, final_norm, lm_head
    (optional for the decoder-only entry point). GEMM weights (w_qkv, w_o, w_router,
    w_gate_up, w_down, lm_head) row-major, packed here into tiled copies; or already tiled
    with packed=True (then pass vocab when the head has no embedding)."""

    PACKED = ("w_qkv", "w_o", "w_router", "w_gate_up", "w_down")

    def __init__(self, layers, head=None, n_q_heads=None, n_kv_heads=None, head_dim=None,
                 top_k=None, rms_eps=1e-6, rope_theta=1e6, packed=False, vocab=None):
        head = dict(head or {})
        if not packed:   # keep tiled copies of the GEMM weights (the caller keeps its own)
            layers = [dict(lw, **{k_: pack_weights(lw[k_]) for k_ in self.PACKED}) for lw in layers]
            if "lm_head" in head:
                head["lm_head"] = pack_weights(head["lm_head"])
        self.layers, self.head = layers, head
        l0 = layers[0]
        E, twoF, d = l0["w_gate_up"].shape
        self.dtype = l0["w_qkv"].dtype
        m = MoltModel()
        m.n_layers = len(layers)
        m.d_model, m.n_q_heads, m.n_kv_heads, m.head_dim = d, n_q_heads, n_kv_heads, head_dim
        m.n_experts, m.top_k, m.d_ff = E, top_k, twoF // 2
        m.vocab = vocab if vocab is not None else (self.head["embed"].shape[0] if "embed" in self.head else 0)
        m.rms_eps, m.rope_theta = rms_eps, rope_theta
        m.dtype = DTYPE_CODE[self.dtype]
        m.expert_dtype = DTYPE_CODE[l0["w_gate_up"].dtype]
        self._arrays = []

        def arr(key, optional=False):
            vals = [lw.get(key) for lw in layers]
            if optional and all(v is None for v in vals):
                return None
            a = (c_vp * len(vals))(*[None if v is None else v.data_ptr() for v in vals])
            self._arrays.append(a)
            return ctypes.cast(a, c_vp)

        for key in ("attn_norm", "w_qkv", "w_o", "moe_norm", "w_router", "w_gate_up", "w_down"):
            setattr(m, key, arr(key))
        for key in ("router_bias", "s_gate_up", "s_down"):
            setattr(m, key, arr(key, optional=True))
        for key in ("embed", "final_norm", "lm_head"):
            setattr(m, key, self.head[key].data_ptr() if key in self.head else None)
        self.struct = m


class KVCache:
    """Per-layer paged caches plus the block tables and context lengths (all on the GPU). Caches of
    kvq_cache (uint8) are 4-bit ones: the calls on a model quantise into them and attend over them."""

    def __init__(self, k_caches, v_caches, block_tables, context_lens):
        self.k_caches, self.v_caches = k_caches, v_caches
        self.block_tables, self.context_lens = block_tables, context_lens
        self._k = (c_vp * len(k_caches))(*[t.data_ptr() for t in k_caches])
        self._v = (c_vp * len(v_caches))(*[t.data_ptr() for t in v_caches])
        s = MoltKV()
        s.k_cache = ctypes.cast(self._k, c_vp)
        s.v_cache = ctypes.cast(self._v, c_vp)
        s.block_tables = block_tables.data_ptr()
        s.context_lens = context_lens.data_ptr()
        s.max_blocks_per_seq = block_tables.shape[1]
        s.num_blocks = k_caches[0].shape[0]
        self.mx = k_caches[0].dtype is torch.uint8
        if any((t.dtype is torch.uint8) != self.mx for t in [*k_caches, *v_caches]):
            raise MoltError("the caches of all layers must be 4-bit ones, or none")
        s.block_size = 16 | MOLT_KV_MX if self.mx else 16
        self.struct = s
        if self.mx:
            self._look_over()

    def _look_over(self):
        """4-bit caches and their tables are whole tensors of one device: a call has addresses only, and would
        take a slice of a pool for its first bytes."""
        named = [(f"{n}[{i}]", t) for n, ts in (("k_caches", self.k_caches), ("v_caches", self.v_caches))
                 for i, t in enumerate(ts)]
        tables = [("block_tables", self.block_tables), ("context_lens", self.context_lens)]
        for name, t in named + tables:
            if not t.is_contiguous():
                raise MoltError(f"{name} must be contiguous (shape {tuple(t.shape)}, strides {t.stride()})")
            if t.get_device() != named[0][1].get_device():
                raise MoltError(f"{name} is on {t.device}, k_caches[0] on {named[0][1].device}")
        for (name, t), dim in zip(tables, (2, 1)):
            if t.dtype is not torch.int32 or t.dim() != dim:
                raise MoltError(f"{name} must be int32 with {dim} dimension(s), is {t.dtype} {tuple(t.shape)}")
        self._shapes = {tuple(t.shape) for _, t in named}

    def check(self, model, B=0):
        """4-bit caches are the model's: its layers and heads, on the current device, tables of B sequences."""
        if not self.mx:
            return
        m = model.struct
        want = (self.struct.num_blocks, m.n_kv_heads, 17 * m.head_dim // 2)
        if self._shapes != {want}:
            raise MoltError(f"a 4-bit cache has shape {[tuple(t.shape) for t in [*self.k_caches, *self.v_caches]]}, "
                            f"expected {want}")
        if not len(self._k) == len(self._v) == m.n_layers:
            raise MoltError(f"{len(self._k)} and {len(self._v)} 4-bit caches for {m.n_layers} layers")
        if min(self.block_tables.shape[0], self.context_lens.shape[0]) < B:
            raise MoltError(f"block_tables has {self.block_tables.shape[0]} rows, context_lens "
                            f"{self.context_lens.shape[0]}, the call has {B} sequences")
        dev = self.k_caches[0].get_device()
        if dev < 0:
            raise MoltError("4-bit caches must be GPU tensors")
        if dev != _current_device():
            raise MoltError(f"the caches are on device {dev}, the current device is {_current_device()}")

    def extra(self, model, B, *ks):
        """Workspace bytes that 4-bit caches add to a call of B sequences of 1 + k positions, for each k of ks."""
        if not self.mx:
            return 0
        self.check(model, B)
        return sum(load().molt_kvq_workspace_extra(ctypes.byref(model.struct), B, k, self.struct.max_blocks_per_seq)
                   for k in ks)


def decoder_workspace_size(model, B, k, max_blocks):
    return load().molt_decoder_workspace_size(ctypes.byref(model.struct), B, k, max_blocks)


def decoder_forward(model, kv, B, k, x, want_routes=False, workspace=None):
    """Runs every layer on the residual stream x [B*(1+k), d] f32 in place."""
    lib = load()
    _dev(x, torch.float32, (B * (k + 1), model.struct.d_model), "x")
    routes = None
    if want_routes:
        routes = torch.empty(model.struct.n_layers, B * (k + 1), model.struct.top_k,
                             dtype=torch.int32, device=x.device)

    def call(ws, nb):
        return lib.molt_decoder_forward(ctypes.byref(model.struct), ctypes.byref(kv.struct), B, k, _ptr(x),
                                        _ptr(routes), ws, nb, _stream())

    _call("molt_decoder_forward", call, decoder_workspace_size(model, B, k, kv.struct.max_blocks_per_seq)
          + kv.extra(model, B, k), x.device, workspace)
    return routes


def verify_step_workspace_size(model, B, k, max_blocks):
    return load().molt_verify_step_workspace_size(ctypes.byref(model.struct), B, k, max_blocks)


def verify_step(model, kv, tokens, uniforms, draft_probs=None, want_logits=True, want_routes=False,
                workspace=None, out=None, want_hidden=False):
    """tokens [B, 1+k] i32. Returns dict(tokens, n_accepted, logprobs, logits?, routes?,
    hidden?) (hidden: the final residual stream [B*(1+k), d] f32, the draft head's input)."""
    lib = load()
    B, kp1 = tokens.shape
    k = kp1 - 1
    V = model.struct.vocab
    dev = tokens.device
    _dev(tokens, torch.int32, name="tokens")
    _dev(uniforms, torch.float32, (B, kp1), "uniforms")
    _dev(draft_probs, torch.float32, (B, k, V), "draft_probs")
    if out is None:
        out = {"tokens": torch.empty(B, kp1, dtype=torch.int32, device=dev),
               "n_accepted": torch.empty(B, dtype=torch.int32, device=dev),
               "logprobs": torch.empty(B, kp1, dtype=torch.float32, device=dev)}
        if want_logits:
            out["logits"] = torch.empty(B, kp1, V, dtype=torch.float32, device=dev)
        if want_routes:
            out["routes"] = torch.empty(model.struct.n_layers, B * kp1, model.struct.top_k,
                                        dtype=torch.int32, device=dev)
        if want_hidden:
            out["hidden"] = torch.empty(B * kp1, model.struct.d_model, dtype=torch.float32, device=dev)

    def call(ws, nb):
        return lib.molt_verify_step(ctypes.byref(model.struct), ctypes.byref(kv.struct), B, k, _ptr(tokens),
                                    _ptr(draft_probs), _ptr(uniforms), _ptr(out.get("logits")),
                                    _ptr(out["tokens"]), _ptr(out["n_accepted"]), _ptr(out["logprobs"]),
                                    _ptr(out.get("routes")), _ptr(out.get("hidden")), ws, nb, _stream())

    _call("molt_verify_step", call, verify_step_workspace_size(model, B, k, kv.struct.max_blocks_per_seq)
          + kv.extra(model, B, k), dev, workspace)
    return out


def prefill_workspace_size(model, B, n, max_blocks):
    return load().molt_prefill_workspace_size(ctypes.byref(model.struct), B, n, max_blocks)


def prefill(model, kv, tokens, lens, want_hidden=False, want_routes=False, workspace=None):
    """Paged prefill (molt_prefill): tokens [B, n] i32 at positions context_lens[b] + j,
    lens [B] i32 in [1, n]. Returns dict(logits [B, V] of each last new row, hidden?, routes?)."""
    lib = load()
    B, n = tokens.shape
    m = model.struct
    dev = tokens.device
    _dev(tokens, torch.int32, name="tokens")
    _dev(lens, torch.int32, (B,), "lens")
    out = {"logits": torch.empty(B, m.vocab, dtype=torch.float32, device=dev)}
    if want_hidden:
        out["hidden"] = torch.empty(B * n, m.d_model, dtype=torch.float32, device=dev)
    if want_routes:
        out["routes"] = torch.empty(m.n_layers, B * n, m.top_k, dtype=torch.int32, device=dev)

    def call(ws, nb):
        return lib.molt_prefill(ctypes.byref(m), ctypes.byref(kv.struct), B, n, _ptr(tokens), _ptr(lens),
                                _ptr(out["logits"]), _ptr(out.get("hidden")), _ptr(out.get("routes")),
                                ws, nb, _stream())

    _call("molt_prefill", call, prefill_workspace_size(model, B, n, kv.struct.max_blocks_per_seq)
          + kv.extra(model, B, n - 1), dev, workspace)
    return out


class PrefixCache:
    """The session-consistent prefix cache (host side, molt_prefix_cache_*): block ids of a
    pool of num_blocks blocks for the callers' block tables. Token lists and rows are host
    (numpy / Python) values."""

    def __init__(self, num_blocks):
        self._lib = load()
        self._c = self._lib.molt_prefix_cache_create(num_blocks)
        if not self._c:
            raise MoltError("molt_prefix_cache_create failed")
        self.num_blocks = num_blocks

    def __del__(self):
        if getattr(self, "_c", None):
            self._lib.molt_prefix_cache_destroy(self._c)
            self._c = None

    def acquire(self, tokens, extra_tokens=0, max_blocks=None):
        """-> (row [n_blocks] int32, n_cached), or None when the pool is exhausted or the row
        would need more than max_blocks blocks."""
        import numpy as np
        toks = np.ascontiguousarray(tokens, dtype=np.int32)
        n = len(toks)
        mb = max_blocks if max_blocks is not None else (n + extra_tokens + 15) // 16
        row = np.empty(max(mb, 1), dtype=np.int32)
        hit = c_int(0)
        r = self._lib.molt_prefix_cache_acquire(self._c, toks.ctypes.data, n, extra_tokens,
                                                row.ctypes.data, mb, ctypes.byref(hit))
        if r < 0:
            return None
        return row[:r].copy(), hit.value

    def commit(self, tokens, row):
        import numpy as np
        toks = np.ascontiguousarray(tokens, dtype=np.int32)
        row = np.ascontiguousarray(row, dtype=np.int32)
        _check(self._lib.molt_prefix_cache_commit(self._c, toks.ctypes.data, len(toks), row.ctypes.data,
                                                  len(row)), "molt_prefix_cache_commit")

    def release(self, row):
        import numpy as np
        row = np.ascontiguousarray(row, dtype=np.int32)
        _check(self._lib.molt_prefix_cache_release(self._c, row.ctypes.data, len(row)),
               "molt_prefix_cache_release")

    def stats(self):
        out = (ctypes.c_longlong * 7)()
        _check(self._lib.molt_prefix_cache_stats(self._c, out), "molt_prefix_cache_stats")
        keys = ("free", "cached", "referenced", "evictable", "lookup_tokens", "hit_tokens", "evictions")
        return dict(zip(keys, list(out)))


def score_tokens_workspace_size(model, B, k, max_blocks):
    return load().molt_score_tokens_workspace_size(ctypes.byref(model.struct), B, k, max_blocks)


def score_tokens(model, kv, tokens, targets, replay_routes=None, want_logits=False, want_routes=False,
                 workspace=None):
    """Behavior-log-prob recompute (molt_score_tokens): tokens, targets [B, 1+k] i32,
    replay_routes [L, B*(1+k), K] i32 or None. Returns dict(logprobs, logits?, routes?)."""
    lib = load()
    B, kp1 = tokens.shape
    k = kp1 - 1
    m = model.struct
    dev = tokens.device
    _dev(tokens, torch.int32, name="tokens")
    _dev(targets, torch.int32, (B, kp1), "targets")
    _dev(replay_routes, torch.int32, (m.n_layers, B * kp1, m.top_k), "replay_routes")
    out = {"logprobs": torch.empty(B, kp1, dtype=torch.float32, device=dev)}
    if want_logits:
        out["logits"] = torch.empty(B, kp1, m.vocab, dtype=torch.float32, device=dev)
    if want_routes:
        out["routes"] = torch.empty(m.n_layers, B * kp1, m.top_k, dtype=torch.int32, device=dev)

    def call(ws, nb):
        return lib.molt_score_tokens(ctypes.byref(m), ctypes.byref(kv.struct), B, k, _ptr(tokens),
                                     _ptr(targets), _ptr(replay_routes), _ptr(out["logprobs"]),
                                     _ptr(out.get("logits")), _ptr(out.get("routes")), ws, nb, _stream())

    _call("molt_score_tokens", call, score_tokens_workspace_size(model, B, k, kv.struct.max_blocks_per_seq)
          + kv.extra(model, B, k), dev, workspace)
    return out


class Mtp:
    """The MTP draft head: enorm, hnorm [d] f32, eh_proj [d, 2d] (row-major; packed here
    into its tiled copy, or already tiled with packed=True), and its decoder layer as a
    one-layer Model whose head holds the output norm (final_norm)."""

    def __init__(self, enorm, hnorm, eh_proj, layer, final_norm, n_q_heads, n_kv_heads, head_dim,
                 top_k, rms_eps=1e-6, rope_theta=1e6, packed=False):
        self.enorm, self.hnorm = enorm, hnorm
        self.eh_proj = eh_proj if packed else pack_weights(eh_proj)
        self.layer = Model([layer], {"final_norm": final_norm}, n_q_heads=n_q_heads,
                           n_kv_heads=n_kv_heads, head_dim=head_dim, top_k=top_k, rms_eps=rms_eps,
                           rope_theta=rope_theta, packed=packed, vocab=0)
        s = MoltMtp()
        s.enorm, s.hnorm, s.eh_proj = enorm.data_ptr(), hnorm.data_ptr(), self.eh_proj.data_ptr()
        s.layer = ctypes.pointer(self.layer.struct)
        self.struct = s


def mtp_draft_workspace_size(target, mtp, B, k, max_blocks, window=None):
    return load().molt_mtp_draft_window_workspace_size(
        ctypes.byref(target.struct), ctypes.byref(mtp.struct), B, k + 1 if window is None else window,
        k, max_blocks)


def mtp_draft(target, mtp, kv, hidden, tokens, n_accepted, next_tokens, uniforms=None,
              greedy=False, k=None, workspace=None, out=None):
    """One draft step (molt_mtp_draft_window): after a verify step (tokens [B, 1+k], the
    default k) or after a prefill (tokens [B, n] = its window, n_accepted = lens - 1, k given).
    hidden [B*W, d] f32, n_accepted [B] i32, next_tokens [B] i32, uniforms [B, k] f32 (unused
    when greedy). Returns dict(drafts [B, k] i32, draft_probs [B, k, V] f32 or None)."""
    lib = load()
    B, W = tokens.shape
    k = W - 1 if k is None else k
    V, d = target.struct.vocab, target.struct.d_model
    dev = tokens.device
    _dev(hidden, torch.float32, (B * W, d), "hidden")
    _dev(tokens, torch.int32, name="tokens")
    _dev(n_accepted, torch.int32, (B,), "n_accepted")
    _dev(next_tokens, torch.int32, (B,), "next_tokens")
    if not greedy:
        _dev(uniforms, torch.float32, (B, k), "uniforms")
    if out is None:
        out = {"drafts": torch.empty(B, k, dtype=torch.int32, device=dev),
               "draft_probs": None if greedy else torch.empty(B, k, V, dtype=torch.float32, device=dev)}

    def call(ws, nb):
        return lib.molt_mtp_draft_window(ctypes.byref(target.struct), ctypes.byref(mtp.struct),
                                         ctypes.byref(kv.struct), B, W, k, _ptr(hidden), _ptr(tokens),
                                         _ptr(n_accepted), _ptr(next_tokens),
                                         _ptr(None if greedy else uniforms), _ptr(out["drafts"]),
                                         _ptr(out["draft_probs"]), ws, nb, _stream())

    _call("molt_mtp_draft", call, mtp_draft_workspace_size(target, mtp, B, k, kv.struct.max_blocks_per_seq, W)
          + kv.extra(mtp.layer, B, W - 1, 0), dev, workspace)
    return out


# ------------------------------------------------------------------ kernel-group timing

PROF_GROUPS = {"attention": 0, "expert_gemm": 1, "lm_head": 2, "sampler": 3, "projections": 4}


def profile_enable(on=True, every=1):
    """on: True (all groups), False (stop), or an iterable of group names to time; every:
    time only launches 0, every, 2 every, ... of each group."""
    if on is True:
        mask = -1
    elif not on:
        mask = 0
    else:
        mask = 0
        for g in on:
            mask |= 1 << PROF_GROUPS[g]
    _check(load().molt_profile_every(every), "molt_profile_every")
    _check(load().molt_profile_enable(mask), "molt_profile_enable")


def profile_read(group):
    """(total milliseconds, number of timed launches) of a kernel group since enable."""
    ms, n = ctypes.c_double(0), c_int(0)
    _check(load().molt_profile_read(PROF_GROUPS[group], ctypes.byref(ms), ctypes.byref(n)),
           "molt_profile_read")
    return ms.value, n.value
