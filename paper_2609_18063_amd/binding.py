"""ctypes binding of libmoe.so (argument marshalling only).

Every function here converts torch tensors to device pointers, passes the
current HIP stream and turns negative return codes into :class:`MoeError`.
All computation happens in the library's HIP kernels.  If the library is
missing, loading fails with ``ImportError``: there is no fallback path.
"""

import ctypes
import sys
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoe.so")

c_int, c_int32, c_int64, c_float, c_void_p, c_size_t = (ctypes.c_int, ctypes.c_int32, ctypes.c_int64,
                                                        ctypes.c_float, ctypes.c_void_p,
                                                        ctypes.c_size_t)

MOE_OK, MOE_EINVAL, MOE_EALIGN, MOE_ENOTRESIDENT, MOE_EHIP, MOE_ENOMEM = 0, -1, -2, -3, -4, -5
MOE_STATUS_SLOT_MISS, MOE_STATUS_BAD_INDEX = 1, 2
MOE_STATUS_BAD_PAGE, MOE_STATUS_BAD_LENGTH = 8, 16
MOE_OUT_F32, MOE_OUT_F16, MOE_OUT_F32_ADD = 0, 1, 2
MOE_ROUTING_SOFTMAX_TOPK, MOE_ROUTING_SIGMOID_GROUP = 0, 1


class MoeLayerSpec(ctypes.Structure):
    _fields_ = [("d_model", c_int32), ("n_experts", c_int32), ("top_k", c_int32),
                ("n_shared", c_int32), ("d_expert", c_int32), ("group_size", c_int32),
                ("lora_rank", c_int32), ("lora_scale", c_float), ("routing", c_int32),
                ("n_groups", c_int32), ("top_groups", c_int32), ("route_scale", c_float),
                ("reserved", c_int32 * 4)]


class MoeProj(ctypes.Structure):
    _fields_ = [("q", c_void_p), ("sz", c_void_p), ("lora_a", c_void_p), ("lora_b", c_void_p)]


class MoeBundle(ctypes.Structure):
    _fields_ = [("gate", MoeProj), ("up", MoeProj), ("down", MoeProj)]


class MoeEngineLayer(ctypes.Structure):
    _fields_ = [("router", c_void_p), ("head", c_void_p), ("mix_d", c_void_p),
                ("mix_perm", c_void_p)]


class MoeHeadMlp(ctypes.Structure):
    _fields_ = [("hidden", c_int32), ("w1_x", c_void_p), ("w1_r", c_void_p), ("b1", c_void_p),
                ("w2", c_void_p), ("b2", c_void_p), ("w_l", c_void_p)]


class MoeBundleLayout(ctypes.Structure):
    _fields_ = [("gate", ctypes.c_int64 * 4), ("up", ctypes.c_int64 * 4),
                ("down", ctypes.c_int64 * 4)]


class MoeStagerStats(ctypes.Structure):
    _fields_ = [("stages", ctypes.c_int64), ("uses", ctypes.c_int64), ("copies", ctypes.c_int64),
                ("bytes", ctypes.c_int64)]


class MoeLatentSpec(ctypes.Structure):
    _fields_ = [("heads", c_int32), ("d_latent", c_int32), ("d_rope", c_int32), ("d_nope", c_int32),
                ("d_v", c_int32), ("page_tokens", c_int32), ("scale", c_float),
                ("reserved", c_int32 * 2)]


class MoeLatentCache(ctypes.Structure):
    _fields_ = [("pages", c_void_p), ("table", c_void_p), ("table_stride", ctypes.c_int64),
                ("n_pages", c_int32), ("n_seqs", c_int32), ("max_pages", c_int32),
                ("reserved", c_int32)]


class MoeError(RuntimeError):
    def __init__(self, code, what):
        self.code = code
        super().__init__("%s failed: %s (%d)" % (what, strerror(code), code))


_lib = None

# name -> (restype, argtypes) for every symbol declared in include/moe_api.h
SIGNATURES = {
    "moe_spec_check": (c_int, [ctypes.POINTER(MoeLayerSpec)]),
    "moe_strerror": (ctypes.c_char_p, [c_int]),
    "moe_slot_table_create": (c_int, [c_int, c_int, c_int, ctypes.POINTER(c_void_p)]),
    "moe_slot_table_destroy": (c_int, [c_void_p]),
    "moe_slot_bind": (c_int, [c_void_p, c_int, c_int, c_int, ctypes.POINTER(MoeBundle)]),
    "moe_slot_unbind": (c_int, [c_void_p, c_int, c_int]),
    "moe_slot_lookup": (c_int, [c_void_p, c_int, c_int]),
    "moe_slot_table_sync": (c_int, [c_void_p, c_void_p]),
    "moe_rmsnorm_f16": (c_int, [c_void_p, c_int, c_int, c_void_p, c_void_p]),
    "moe_workspace_bytes": (c_size_t, [ctypes.POINTER(MoeLayerSpec), c_int]),
    "moe_route": (c_int, [ctypes.POINTER(MoeLayerSpec), c_void_p, c_void_p, c_int, c_void_p,
                          c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "moe_preroute": (c_int, [ctypes.POINTER(MoeLayerSpec), c_void_p, c_void_p, c_int, c_void_p,
                             c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "moe_preroute_mlp_workspace_bytes": (c_size_t, [ctypes.POINTER(MoeLayerSpec), c_int, c_int]),
    "moe_preroute_mlp": (c_int, [ctypes.POINTER(MoeLayerSpec), ctypes.POINTER(MoeHeadMlp), c_void_p,
                                 c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                 c_size_t, c_void_p]),
    "moe_expert_ffn_int4_lora": (c_int, [ctypes.POINTER(MoeLayerSpec), c_void_p, c_int, c_void_p,
                                         c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t,
                                         c_void_p]),
    "moe_expert_ffn_int4_lora_noalloc": (c_int, [ctypes.POINTER(MoeLayerSpec), c_void_p, c_int,
                                                 c_void_p, c_int, c_void_p, c_void_p, c_void_p,
                                                 c_void_p]),
    "moe_expert_ffn_grouped_int4_lora": (c_int, [ctypes.POINTER(MoeLayerSpec), c_void_p, c_int,
                                                 c_void_p, c_int, c_void_p, c_void_p, c_void_p,
                                                 c_void_p, c_size_t, c_void_p]),
    "moe_combine": (c_int, [ctypes.POINTER(MoeLayerSpec), c_void_p, c_void_p, c_int, c_void_p,
                            c_void_p]),
    "moe_topk": (c_int, [ctypes.POINTER(MoeLayerSpec), c_void_p, c_int, c_void_p, c_void_p,
                         c_void_p]),
    "moe_topk_biased": (c_int, [ctypes.POINTER(MoeLayerSpec), c_void_p, c_void_p, c_int, c_void_p,
                                c_void_p, c_void_p]),
    "moe_profile_arm": (c_int, [c_int, c_void_p, c_void_p]),
    "moe_merge_requantize": (c_int, [ctypes.POINTER(MoeProj), c_int, c_int, c_int, ctypes.c_float,
                                     c_void_p, c_void_p, c_void_p, c_void_p]),
    "moe_slot_policy_create": (c_int, [c_int, c_int, c_int, ctypes.POINTER(c_void_p)]),
    "moe_slot_policy_destroy": (c_int, [c_void_p]),
    "moe_slot_policy_stage": (c_int, [c_void_p, c_int, c_void_p, c_int, c_void_p]),
    "moe_slot_policy_use": (c_int, [c_void_p, c_int, c_void_p, c_int, c_void_p]),
    "moe_slot_policy_release": (c_int, [c_void_p, c_int]),
    "moe_slot_policy_lookup": (c_int, [c_void_p, c_int, c_int]),
    "moe_stager_create": (c_int, [c_void_p, ctypes.POINTER(MoeBundleLayout), c_size_t, c_void_p,
                                  c_void_p, c_size_t, ctypes.POINTER(c_void_p)]),
    "moe_stager_destroy": (c_int, [c_void_p]),
    "moe_stager_create_file": (c_int, [c_void_p, ctypes.POINTER(MoeBundleLayout), c_size_t,
                                       ctypes.c_char_p, c_size_t, c_int, c_int, c_void_p, c_size_t,
                                       ctypes.POINTER(c_void_p)]),
    "moe_stager_io_stats": (c_int, [c_void_p, ctypes.POINTER(ctypes.c_int64),
                                    ctypes.POINTER(ctypes.c_int64)]),
    "moe_stager_stage": (c_int, [c_void_p, c_int, c_void_p, c_int, c_void_p, c_void_p]),
    "moe_stager_use": (c_int, [c_void_p, c_int, c_void_p, c_int, c_void_p, c_void_p]),
    "moe_stager_release": (c_int, [c_void_p, c_int]),
    "moe_stager_stats_get": (c_int, [c_void_p, ctypes.POINTER(MoeStagerStats)]),
    "moe_combine_add": (c_int, [ctypes.POINTER(MoeLayerSpec), c_void_p, c_void_p, c_int, c_void_p,
                                c_void_p]),
    "moe_chain_token_start": (c_int, [c_void_p, c_int, c_void_p, c_void_p]),
    "moe_chain_mix_rmsnorm": (c_int, [c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_void_p]),
    "moe_linear_workspace_bytes": (c_size_t, [c_int, c_int, c_int, c_int]),
    "moe_linear_int4_lora": (c_int, [ctypes.POINTER(MoeProj), c_int, c_int, c_int, c_float, c_void_p,
                                     c_int64, c_int, c_void_p, c_int, c_int64, c_void_p, c_size_t,
                                     c_void_p]),
    "moe_latent_spec_check": (c_int, [ctypes.POINTER(MoeLatentSpec)]),
    "moe_latent_append": (c_int, [ctypes.POINTER(MoeLatentSpec), ctypes.POINTER(MoeLatentCache), c_void_p,
                                  c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_int, c_void_p,
                                  c_void_p, c_void_p, c_void_p]),
    "moe_latent_decode_workspace_bytes": (c_size_t, [ctypes.POINTER(MoeLatentSpec), c_int, c_int, c_int]),
    "moe_latent_decode": (c_int, [ctypes.POINTER(MoeLatentSpec), ctypes.POINTER(MoeLatentCache), c_void_p,
                                  c_void_p, c_int, c_void_p, c_int, c_void_p, c_int, c_void_p, c_void_p,
                                  c_void_p, c_size_t, c_void_p]),
    "moe_latent_prefill_workspace_bytes": (c_size_t, [ctypes.POINTER(MoeLatentSpec), c_int, c_int]),
    "moe_latent_prefill": (c_int, [ctypes.POINTER(MoeLatentSpec), ctypes.POINTER(MoeLatentCache), c_void_p,
                                   c_void_p, c_int, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p,
                                   c_void_p, c_void_p, c_size_t, c_void_p]),
    "moe_latent4_page_bytes": (c_size_t, [ctypes.POINTER(MoeLatentSpec)]),
    "moe_latent4_append": (c_int, [ctypes.POINTER(MoeLatentSpec), ctypes.POINTER(MoeLatentCache), c_void_p,
                                   c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_void_p, c_int, c_void_p,
                                   c_void_p, c_void_p, c_void_p]),
    "moe_latent4_read": (c_int, [ctypes.POINTER(MoeLatentSpec), ctypes.POINTER(MoeLatentCache), c_void_p,
                                 c_void_p, c_int, c_void_p, c_void_p, c_void_p]),
    "moe_latent4_decode_workspace_bytes": (c_size_t, [ctypes.POINTER(MoeLatentSpec), c_int, c_int, c_int]),
    "moe_latent4_decode": (c_int, [ctypes.POINTER(MoeLatentSpec), ctypes.POINTER(MoeLatentCache), c_void_p,
                                   c_void_p, c_int, c_void_p, c_int, c_void_p, c_void_p, c_int64, c_void_p,
                                   c_void_p, c_size_t, c_void_p]),
    "moe_latent4_prefill_workspace_bytes": (c_size_t, [ctypes.POINTER(MoeLatentSpec), c_int, c_int, c_int,
                                                       c_int]),
    "moe_latent4_prefill": (c_int, [ctypes.POINTER(MoeLatentSpec), ctypes.POINTER(MoeLatentCache), c_void_p,
                                    c_void_p, c_int, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p,
                                    c_void_p, c_int64, c_int, c_void_p, c_void_p, c_size_t, c_void_p]),
    "moe_evict_select": (c_int, [c_void_p, c_void_p, c_int, c_int, c_int, c_void_p, c_int, c_int, c_int,
                                 c_void_p, c_void_p, c_void_p]),
    "moe_latent4_move": (c_int, [ctypes.POINTER(MoeLatentSpec), ctypes.POINTER(MoeLatentCache), c_int, c_int64,
                                 c_void_p, c_int, c_int, c_void_p, c_int64, c_void_p, c_void_p]),
    "moe_page_pool_create": (c_int, [c_int, c_int, ctypes.POINTER(c_void_p)]),
    "moe_page_pool_destroy": (c_int, [c_void_p]),
    "moe_page_pool_available": (c_int, [c_void_p]),
    "moe_page_pool_refs": (c_int, [c_void_p, c_int]),
    "moe_page_pool_alloc": (c_int, [c_void_p, c_int, c_void_p]),
    "moe_page_pool_fork": (c_int, [c_void_p, c_void_p, c_int64, c_void_p, c_void_p]),
    "moe_page_pool_free": (c_int, [c_void_p, c_void_p, c_int]),
    "moe_page_pool_compact": (c_int, [c_void_p, c_void_p, c_void_p]),
    "moe_page_copy": (c_int, [c_void_p, c_int, c_int64, c_int64, c_int, c_void_p, c_int, c_void_p,
                              c_void_p]),
    "moe_page_remap": (c_int, [c_void_p, c_int64, c_void_p, c_int, c_void_p, c_void_p, c_void_p]),
    "moe_engine_supported": (c_int, [ctypes.POINTER(MoeLayerSpec)]),
    "moe_engine_workspace_bytes": (c_size_t, [ctypes.POINTER(MoeLayerSpec), c_int]),
    "moe_engine_layers": (c_int, [ctypes.POINTER(MoeLayerSpec), c_void_p, c_void_p, c_void_p, c_int,
                                  c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                  c_void_p, c_void_p, c_size_t, c_void_p]),
    "moe_engine_tokens_supported": (c_int, [ctypes.POINTER(MoeLayerSpec)]),
    "moe_engine_tokens": (c_int, [ctypes.POINTER(MoeLayerSpec), c_void_p, c_void_p, c_void_p, c_int,
                                  c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                  c_void_p, c_void_p, c_size_t, c_void_p]),
    "moe_engine_chain_supported": (c_int, [ctypes.POINTER(MoeLayerSpec)]),
    "moe_engine_chain_mlp_supported": (c_int, [ctypes.POINTER(MoeLayerSpec), c_int]),
    "moe_engine_chain_mlp": (c_int, [ctypes.POINTER(MoeLayerSpec), c_void_p, c_void_p, c_void_p, c_int, c_int,
                                     c_int, c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                     c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, ctypes.c_size_t,
                                     c_void_p]),
    "moe_engine_chain": (c_int, [ctypes.POINTER(MoeLayerSpec), c_void_p, c_void_p, c_int, c_int,
                                 c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                 c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t,
                                 c_void_p]),
}

MOE_PROF_FFN_MAIN = 0
MOE_PROF_ENGINE_PHASES = 1


def lib():
    """Load libmoe.so once and declare its signatures."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libmoe.so is not built (%s); run __graft_entry__.build()" % LIB_PATH)
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype, fn.argtypes = res, args
        _lib = handle
    return _lib


def strerror(code):
    return lib().moe_strerror(int(code)).decode()


def _check(rc, what):
    if rc < 0:
        raise MoeError(rc, what)
    return rc


# A call at T = 1 costs the host more than the GPU (its kernels are a few us each), so
# addresses go to ctypes as plain integers and the current stream is read without
# building a Stream object.

def _ptr(t):
    return None if t is None else t.data_ptr()


_torch = None
_raw_stream = None


def _public_stream():
    return _torch.cuda.current_stream().cuda_stream


def _stream_reader():
    """How the current stream is read: torch's internal reader (0.2 us a call; 3.1 us
    through a Stream object) where this torch has it and it agrees with the public one."""
    c = _torch._C
    try:
        raw, device = c._cuda_getCurrentRawStream, c._cuda_getDevice
        if raw(device()) == _public_stream():
            return lambda: raw(device())
    except (AttributeError, TypeError):
        pass
    return _public_stream


def _stream(stream=None):
    global _torch, _raw_stream
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        if _torch is None:
            import torch
            _torch = torch
        if not _torch.cuda.is_initialized():
            return _public_stream()
        _raw_stream = _stream_reader()
    return _raw_stream()


class StreamPair:
    """Two streams for work that must overlap (copies beside kernels), taken
    one right after the other from torch's stream pool (default priority).
    The pool creates its streams together, and HIP maps streams onto a few
    hardware queues (GPU_MAX_HW_QUEUES) in creation order, so consecutive pool
    streams sit on different queues; a pool stream paired with the null
    stream can share its queue and serialize against it. Pool streams live as
    long as the process, so ``close`` has nothing to free."""

    def __init__(self):
        import torch
        self.compute = torch.cuda.Stream()
        self.copy = torch.cuda.Stream()

    def close(self):
        pass


def make_spec(d, n_experts, top_k, n_shared, d_expert, lora_rank, lora_scale, group_size=64,
              sigmoid_group=None):
    """``sigmoid_group``: None (softmax-topk) or (n_groups, top_groups, scale)."""
    s = MoeLayerSpec()
    s.d_model, s.n_experts, s.top_k, s.n_shared = d, n_experts, top_k, n_shared
    s.d_expert, s.group_size, s.lora_rank, s.lora_scale = d_expert, group_size, lora_rank, lora_scale
    s.routing = MOE_ROUTING_SOFTMAX_TOPK
    if sigmoid_group is not None:
        s.routing = MOE_ROUTING_SIGMOID_GROUP
        s.n_groups, s.top_groups, s.route_scale = sigmoid_group
    return s


def spec_from_workload(wl):
    return make_spec(wl.d, wl.E, wl.K, wl.S, wl.I, wl.r, wl.lora_scale)


def spec_check(spec):
    return lib().moe_spec_check(ctypes.byref(spec))


def workspace_bytes(spec, T):
    return int(lib().moe_workspace_bytes(ctypes.byref(spec), int(T)))


class SlotTable:
    """Owner of a library slot table (host mirror + device copy)."""

    def __init__(self, n_layers, n_ids, n_slots):
        h = c_void_p()
        _check(lib().moe_slot_table_create(n_layers, n_ids, n_slots, ctypes.byref(h)),
               "moe_slot_table_create")
        self.handle = h
        self.n_layers, self.n_ids, self.n_slots = n_layers, n_ids, n_slots
        self._keep = {}

    def bind(self, layer, expert, slot, bundle, keep=None):
        _check(lib().moe_slot_bind(self.handle, layer, expert, slot, ctypes.byref(bundle)),
               "moe_slot_bind")
        self._keep[(layer, slot)] = keep

    def unbind(self, layer, expert):
        _check(lib().moe_slot_unbind(self.handle, layer, expert), "moe_slot_unbind")

    def lookup(self, layer, expert):
        rc = lib().moe_slot_lookup(self.handle, layer, expert)
        if rc == MOE_ENOTRESIDENT:
            return -1
        return _check(rc, "moe_slot_lookup")

    def sync(self, stream=None):
        _check(lib().moe_slot_table_sync(self.handle, _stream(stream)), "moe_slot_table_sync")

    def close(self):
        if self.handle:
            _check(lib().moe_slot_table_destroy(self.handle), "moe_slot_table_destroy")
            self.handle = None

    def __del__(self, _finalizing=sys.is_finalizing):
        # no runtime calls while the interpreter shuts down: close() explicitly
        if _finalizing():
            return
        try:
            self.close()
        except Exception:
            pass


def _i32(a):
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


class SlotPolicy:
    """The library's host-tier slot policy (host logic only)."""

    def __init__(self, n_layers, n_ids, n_slots):
        h = c_void_p()
        _check(lib().moe_slot_policy_create(n_layers, n_ids, n_slots, ctypes.byref(h)),
               "moe_slot_policy_create")
        self.handle = h

    def stage(self, layer, experts):
        e = _i32(experts)
        out = np.zeros((max(len(e), 1), 2), dtype=np.int32)
        n = _check(lib().moe_slot_policy_stage(self.handle, layer, e.ctypes.data, len(e),
                                               out.ctypes.data), "moe_slot_policy_stage")
        return [tuple(int(v) for v in out[i]) for i in range(n)]

    def use(self, layer, experts):
        e = _i32(experts)
        out = np.zeros(max(len(e), 1), dtype=np.int32)
        _check(lib().moe_slot_policy_use(self.handle, layer, e.ctypes.data, len(e), out.ctypes.data),
               "moe_slot_policy_use")
        return out[:len(e)].tolist()

    def release(self, layer):
        _check(lib().moe_slot_policy_release(self.handle, layer), "moe_slot_policy_release")

    def lookup(self, layer, expert):
        rc = lib().moe_slot_policy_lookup(self.handle, layer, expert)
        return -1 if rc == MOE_ENOTRESIDENT else _check(rc, "moe_slot_policy_lookup")

    def close(self):
        if self.handle:
            lib().moe_slot_policy_destroy(self.handle)
            self.handle = None

    def __del__(self, _finalizing=sys.is_finalizing):
        # no runtime calls while the interpreter shuts down: close() explicitly
        if _finalizing():
            return
        try:
            self.close()
        except Exception:
            pass


class Stager:
    """The slot policy driving a slot table: pinned host bundles -> device slots."""

    def __init__(self, table, layout, bundle_bytes, host_ptrs, slot_pool, slot_stride, file=None):
        """``file``: None (bundles at ``host_ptrs`` in pinned memory) or
        ``(path, file_stride, n_bounce, n_io)`` for the file tier."""
        h = c_void_p()
        if file is None:
            ptrs = (c_void_p * len(host_ptrs))(*host_ptrs)
            _check(lib().moe_stager_create(table.handle, ctypes.byref(layout), bundle_bytes, ptrs,
                                           _ptr(slot_pool), slot_stride, ctypes.byref(h)),
                   "moe_stager_create")
        else:
            path, file_stride, n_bounce, n_io = file
            _check(lib().moe_stager_create_file(table.handle, ctypes.byref(layout), bundle_bytes,
                                                str(path).encode(), file_stride, n_bounce, n_io,
                                                _ptr(slot_pool), slot_stride, ctypes.byref(h)),
                   "moe_stager_create_file")
        self.handle = h
        self.table, self.pool = table, slot_pool

    def io_stats(self):
        ns, nb = ctypes.c_int64(), ctypes.c_int64()
        _check(lib().moe_stager_io_stats(self.handle, ctypes.byref(ns), ctypes.byref(nb)),
               "moe_stager_io_stats")
        return {"read_ns": ns.value, "read_bytes": nb.value}

    def stage(self, layer, experts, copy_stream):
        e = _i32(experts)
        out = np.zeros((max(len(e), 1), 2), dtype=np.int32)
        n = _check(lib().moe_stager_stage(self.handle, layer, e.ctypes.data, len(e),
                                          ctypes.c_void_p(copy_stream.cuda_stream),
                                          out.ctypes.data), "moe_stager_stage")
        return [tuple(int(v) for v in out[i]) for i in range(n)]

    def use(self, layer, experts, compute_stream=None):
        e = _i32(experts)
        out = np.zeros(max(len(e), 1), dtype=np.int32)
        _check(lib().moe_stager_use(self.handle, layer, e.ctypes.data, len(e),
                                    _stream(compute_stream), out.ctypes.data), "moe_stager_use")
        return out[:len(e)].tolist()

    def release(self, layer):
        _check(lib().moe_stager_release(self.handle, layer), "moe_stager_release")

    def stats(self):
        st = MoeStagerStats()
        _check(lib().moe_stager_stats_get(self.handle, ctypes.byref(st)), "moe_stager_stats_get")
        return {"stages": st.stages, "uses": st.uses, "copies": st.copies, "bytes": st.bytes}

    def close(self):
        if self.handle:
            lib().moe_stager_destroy(self.handle)
            self.handle = None

    def __del__(self, _finalizing=sys.is_finalizing):
        # no runtime calls while the interpreter shuts down: close() explicitly
        if _finalizing():
            return
        try:
            self.close()
        except Exception:
            pass


# ---- weights: host arrays in the stored format -> device buffers --------------

def upload_projection(qsz, lora, device):
    """(packed q [out, in/2] uint8, s fp16 [out, in/64], z fp16) + (A, B) | None
    -> (MoeProj, tensors to keep alive).  s and z are interleaved into the
    (scale, zero) pairs of the device layout."""
    import torch
    q, s, z = qsz
    qt = torch.from_numpy(np.ascontiguousarray(q)).to(device)
    sz = np.ascontiguousarray(np.stack([np.asarray(s, np.float16), np.asarray(z, np.float16)], -1))
    szt = torch.from_numpy(sz).to(device)
    keep = [qt, szt]
    p = MoeProj(qt.data_ptr(), szt.data_ptr(), None, None)
    if lora is not None:
        at = torch.from_numpy(np.ascontiguousarray(lora[0], dtype=np.float16)).to(device)
        bt = torch.from_numpy(np.ascontiguousarray(lora[1], dtype=np.float16)).to(device)
        keep += [at, bt]
        p.lora_a, p.lora_b = at.data_ptr(), bt.data_ptr()
    return p, keep


def upload_bundle(b, device="cuda"):
    lo = b.get("lora") or {}
    g, kg = upload_projection(b["gate"], lo.get("gate"), device)
    u, ku = upload_projection(b["up"], lo.get("up"), device)
    d, kd = upload_projection(b["down"], lo.get("down"), device)
    return MoeBundle(g, u, d), kg + ku + kd


# ---- hot path -----------------------------------------------------------------

def rmsnorm_f16(xi, x, stream=None):
    T, d = xi.shape
    _check(lib().moe_rmsnorm_f16(_ptr(xi), T, d, _ptr(x), _stream(stream)), "moe_rmsnorm_f16")


def route(spec, x, w_router, idx, w, workspace, logits=None, stream=None):
    T = x.shape[0]
    _check(lib().moe_route(ctypes.byref(spec), _ptr(x), _ptr(w_router), T, _ptr(logits), _ptr(idx),
                           _ptr(w), _ptr(workspace), workspace.nbytes,
                           _stream(stream)), "moe_route")


def preroute(spec_next, x, w_head, pred_idx, pred_w, workspace, logits=None, stream=None):
    T = x.shape[0]
    _check(lib().moe_preroute(ctypes.byref(spec_next), _ptr(x), _ptr(w_head), T, _ptr(logits),
                              _ptr(pred_idx), _ptr(pred_w), _ptr(workspace),
                              workspace.nbytes, _stream(stream)),
           "moe_preroute")


def head_mlp(hidden, w1_x, w1_r, w2, b1=None, b2=None, w_l=None):
    """moe_head_mlp of device fp16 tensors (layouts as in include/moe_api.h)."""
    def p(t):
        return None if t is None else t.data_ptr()
    return MoeHeadMlp(hidden, p(w1_x), p(w1_r), p(b1), p(w2), p(b2), p(w_l))


def preroute_mlp_workspace_bytes(spec_next, hidden, T):
    return lib().moe_preroute_mlp_workspace_bytes(ctypes.byref(spec_next), hidden, T)


def preroute_mlp(spec_next, head, x, routed_t, routed_tm1, pred_idx, pred_w, workspace, logits=None,
                 stream=None):
    """Full prerouter head (moe_preroute_mlp); ``head`` from ``head_mlp``."""
    T = x.shape[0]
    _check(lib().moe_preroute_mlp(ctypes.byref(spec_next), ctypes.byref(head), _ptr(x), T, _ptr(routed_t),
                                  _ptr(routed_tm1), _ptr(logits), _ptr(pred_idx), _ptr(pred_w),
                                  _ptr(workspace), workspace.nbytes,
                                  _stream(stream)), "moe_preroute_mlp")


def expert_ffn(spec, table, layer, x, idx, y_experts, status, workspace, stream=None):
    T = x.shape[0]
    _check(lib().moe_expert_ffn_int4_lora(ctypes.byref(spec), table.handle, layer, _ptr(x), T,
                                          _ptr(idx), _ptr(y_experts), _ptr(status), _ptr(workspace),
                                          workspace.nbytes,
                                          _stream(stream)), "moe_expert_ffn_int4_lora")


MOE_NOALLOC_SCRATCH_BYTES = 4 << 20


def expert_ffn_noalloc(spec, table, layer, x, idx, y_experts, status, stream=None):
    """``expert_ffn`` without a workspace: the library's static per-device scratch."""
    T = x.shape[0]
    _check(lib().moe_expert_ffn_int4_lora_noalloc(ctypes.byref(spec), table.handle, layer, _ptr(x),
                                                  T, _ptr(idx), _ptr(y_experts), _ptr(status),
                                                  _stream(stream)),
           "moe_expert_ffn_int4_lora_noalloc")


def expert_ffn_grouped(spec, table, layer, x, idx, y_experts, status, workspace, stream=None):
    """Batched / prefill experts: same contract as ``expert_ffn``, grouped by expert."""
    T = x.shape[0]
    _check(lib().moe_expert_ffn_grouped_int4_lora(ctypes.byref(spec), table.handle, layer, _ptr(x),
                                                  T, _ptr(idx), _ptr(y_experts), _ptr(status),
                                                  _ptr(workspace),
                                                  workspace.nbytes,
                                                  _stream(stream)),
           "moe_expert_ffn_grouped_int4_lora")


def combine(spec, y_experts, w, y, stream=None):
    T = y.shape[0]
    _check(lib().moe_combine(ctypes.byref(spec), _ptr(y_experts), _ptr(w), T, _ptr(y),
                             _stream(stream)), "moe_combine")


def topk(spec, logits, idx, w, stream=None):
    T = logits.shape[0]
    _check(lib().moe_topk(ctypes.byref(spec), _ptr(logits), T, _ptr(idx), _ptr(w), _stream(stream)),
           "moe_topk")


def topk_biased(spec, logits, bias, idx, w, stream=None):
    """Sigmoid-group top-k with a selection bias (fp32 [E] device tensor or None)."""
    T = logits.shape[0]
    _check(lib().moe_topk_biased(ctypes.byref(spec), _ptr(logits), _ptr(bias), T, _ptr(idx), _ptr(w),
                                 _stream(stream)), "moe_topk_biased")


def merge_requantize(proj, out_dim, in_dim, rank, lora_scale, q_out, sz_out, stats=None,
                     stream=None):
    """moe_merge_requantize: ``proj`` a MoeProj of device pointers; ``q_out``
    uint8 ``[out, in/2]``, ``sz_out`` fp16 ``[out, in/64, 2]``, ``stats``
    float64 ``[out, in/64, 2]`` or None (device tensors)."""
    _check(lib().moe_merge_requantize(ctypes.byref(proj), out_dim, in_dim, rank, lora_scale,
                                      _ptr(q_out), _ptr(sz_out), _ptr(stats), _stream(stream)),
           "moe_merge_requantize")


def profile_arm(which, start_event, stop_event):
    """Time the next launch of kernel ``which`` with two hipEvent_t handles (ints)."""
    _check(lib().moe_profile_arm(which, ctypes.c_void_p(start_event), ctypes.c_void_p(stop_event)),
           "moe_profile_arm")


def combine_add(spec, y_experts, w, y_inout, stream=None):
    T = y_inout.shape[0]
    _check(lib().moe_combine_add(ctypes.byref(spec), _ptr(y_experts), _ptr(w), T, _ptr(y_inout),
                                 _stream(stream)), "moe_combine_add")


def chain_token_start(xi, r, stream=None):
    _check(lib().moe_chain_token_start(_ptr(xi), r.numel(), _ptr(r), _stream(stream)),
           "moe_chain_token_start")


def chain_mix_rmsnorm(mix_d, perm, r, x, stream=None):
    _check(lib().moe_chain_mix_rmsnorm(_ptr(mix_d), _ptr(perm), r.numel(), _ptr(r), _ptr(x),
                                       _stream(stream)), "moe_chain_mix_rmsnorm")


MOE_STATUS_ENGINE_ABORT = 4


def engine_supported(spec):
    return lib().moe_engine_supported(ctypes.byref(spec)) == MOE_OK


def engine_chain_supported(spec):
    return lib().moe_engine_chain_supported(ctypes.byref(spec)) == MOE_OK


def engine_workspace_bytes(spec, n_layers):
    return int(lib().moe_engine_workspace_bytes(ctypes.byref(spec), int(n_layers)))


def engine_chain_mlp_supported(spec, hidden):
    return lib().moe_engine_chain_mlp_supported(ctypes.byref(spec), int(hidden)) == MOE_OK


def head_mlp_array(heads, device="cuda"):
    """Device array of moe_head_mlp (one per layer; None entries -> all NULL)."""
    import torch
    arr = (MoeHeadMlp * len(heads))()
    for i, h in enumerate(heads):
        if h is not None:
            arr[i] = h
    raw = np.frombuffer(bytes(arr), dtype=np.uint8).copy()
    return torch.from_numpy(raw).to(device)


def engine_layer_array(layers, device="cuda"):
    """Device array of moe_engine_layer from dicts of device tensors
    (router, head, mix_d, mix_perm; missing or None -> NULL)."""
    import torch
    arr = (MoeEngineLayer * len(layers))()
    for i, lay in enumerate(layers):
        def p(k):
            t = lay.get(k)
            return None if t is None else t.data_ptr()
        arr[i] = MoeEngineLayer(p("router"), p("head"), p("mix_d"), p("mix_perm"))
    raw = np.frombuffer(bytes(arr), dtype=np.uint8).copy()
    return torch.from_numpy(raw).to(device)


def engine_layers(spec, table, layer_arr, step_layer, xi, y, workspace, idx=None, w=None,
                  pidx=None, pw=None, status=None, stream=None):
    n = step_layer.numel()
    _check(lib().moe_engine_layers(ctypes.byref(spec), table.handle, _ptr(layer_arr),
                                   _ptr(step_layer), n, _ptr(xi), _ptr(y), _ptr(idx), _ptr(w),
                                   _ptr(pidx), _ptr(pw), _ptr(status), _ptr(workspace),
                                   workspace.nbytes, _stream(stream)),
           "moe_engine_layers")


def engine_tokens_supported(spec):
    return lib().moe_engine_tokens_supported(ctypes.byref(spec)) == MOE_OK


def engine_tokens(spec, table, layer_arr, step_layer, xi, y, workspace, idx=None, w=None,
                  pidx=None, pw=None, status=None, stream=None):
    """moe_engine_tokens: the steps of engine_layers, one per team of 16 workgroups in flight."""
    n = step_layer.numel()
    _check(lib().moe_engine_tokens(ctypes.byref(spec), table.handle, _ptr(layer_arr),
                                   _ptr(step_layer), n, _ptr(xi), _ptr(y), _ptr(idx), _ptr(w),
                                   _ptr(pidx), _ptr(pw), _ptr(status), _ptr(workspace),
                                   workspace.nbytes, _stream(stream)),
           "moe_engine_tokens")


def engine_chain(spec, table, layer_arr, n_layers, first_token, xi, r_state, workspace,
                 x_rec=None, idx=None, w=None, pidx=None, pw=None, y_rec=None, status=None,
                 stream=None, r_rec=None):
    n_tokens = xi.shape[0]
    _check(lib().moe_engine_chain(ctypes.byref(spec), table.handle, _ptr(layer_arr), n_layers,
                                  first_token, n_tokens, _ptr(xi), _ptr(r_state), _ptr(x_rec),
                                  _ptr(r_rec), _ptr(idx), _ptr(w), _ptr(pidx), _ptr(pw),
                                  _ptr(y_rec),
                                  _ptr(status), _ptr(workspace),
                                  workspace.nbytes, _stream(stream)),
           "moe_engine_chain")


def engine_chain_mlp(spec, table, layer_arr, head_arr, hidden, n_layers, first_token, xi, r_state, workspace,
                     x_rec=None, idx=None, w=None, pidx=None, pw=None, y_rec=None, status=None,
                     stream=None, r_rec=None):
    """moe_engine_chain_mlp: the chain with the full prerouter head of every
    layer (head_arr from head_mlp_array)."""
    n_tokens = xi.shape[0]
    _check(lib().moe_engine_chain_mlp(ctypes.byref(spec), table.handle, _ptr(layer_arr), _ptr(head_arr),
                                      int(hidden), n_layers, first_token, n_tokens, _ptr(xi), _ptr(r_state),
                                      _ptr(x_rec), _ptr(r_rec), _ptr(idx), _ptr(w), _ptr(pidx), _ptr(pw),
                                      _ptr(y_rec), _ptr(status), _ptr(workspace),
                                      workspace.nbytes, _stream(stream)),
           "moe_engine_chain_mlp")


# ---- attention block --------------------------------------------------------------

def _need(ok, what):
    if not ok:
        raise ValueError(what)


_device = None


def _the_torch():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _current_device():
    """The current GPU, by torch's internal reader where it has one (0.06 us a call; 0.3 us through torch.cuda)."""
    global _device
    if _device is None:
        t = _the_torch()
        if not t.cuda.is_available():
            return -2                                    # (no tensor is there; -1 is the CPU)
        t.cuda.current_device()                          # (the internal one needs what this sets up)
        _device = getattr(t._C, "_cuda_getDevice", t.cuda.current_device)
    return _device()


def _dense(what, dtype, *tensors):
    """Contiguous tensors of one dtype on the current GPU (None: left out): the library sees addresses only, and
    launches there."""
    here = _current_device()
    for t in tensors:
        if t is None:
            continue
        if t.dtype != dtype or not t.is_contiguous() or t.get_device() != here:
            raise ValueError("%s: a contiguous %s tensor on the current GPU is needed, got %s %s on %s"
                             % (what, dtype, t.dtype, tuple(t.stride()), t.device))


def _room(workspace):
    _dense("workspace", workspace.dtype, workspace)


def linear_workspace_bytes(out_dim, in_dim, rank, T):
    return int(lib().moe_linear_workspace_bytes(out_dim, in_dim, rank, T))


def linear_int4(proj, out_dim, in_dim, rank, lora_scale, x, y, workspace, add=False, stream=None):
    """moe_linear_int4_lora: ``proj`` a MoeProj of device pointers; ``x`` fp16 ``[T, in]`` and ``y`` fp32 or
    fp16 ``[T, out]`` with unit column stride; ``add``: into an fp32 ``y``."""
    torch = _the_torch()
    T = x.shape[0]
    f16 = y.dtype == torch.float16
    _need(x.dtype == torch.float16 and x.dim() == 2 and x.shape[1] == in_dim and (in_dim == 1 or x.stride(1) == 1),
          "x: fp16 [T, in] with unit column stride")
    _need((f16 or y.dtype == torch.float32) and y.shape == (T, out_dim) and (out_dim == 1 or y.stride(1) == 1),
          "y: fp32 or fp16 [T, out] with unit column stride")
    _need(not (add and f16), "add needs an fp32 y")
    _room(workspace)
    _need(x.device == y.device == workspace.device, "x, y and the workspace on one GPU")
    _check(lib().moe_linear_int4_lora(ctypes.byref(proj), out_dim, in_dim, rank, lora_scale, _ptr(x),
                                      x.stride(0) if T > 1 else in_dim, T, _ptr(y),
                                      MOE_OUT_F16 if f16 else MOE_OUT_F32_ADD if add else MOE_OUT_F32,
                                      y.stride(0) if T > 1 else out_dim, _ptr(workspace), workspace.nbytes,
                                      _stream(stream)), "moe_linear_int4_lora")


def make_latent_spec(heads, d_latent, d_rope, d_nope, d_v, page_tokens, scale):
    s = MoeLatentSpec()
    s.heads, s.d_latent, s.d_rope, s.d_nope, s.d_v = heads, d_latent, d_rope, d_nope, d_v
    s.page_tokens, s.scale = page_tokens, scale
    return s


def latent_spec_check(spec):
    return lib().moe_latent_spec_check(ctypes.byref(spec))


def latent_cache(pages, table):
    """moe_latent_cache of ``pages`` fp16 ``[n_pages, page_tokens, d_latent + d_rope]`` and ``table`` int32
    ``[n_seqs, max_pages]`` (rows may be strided). The struct keeps both alive."""
    _dense("pages", _the_torch().float16, pages)
    _need(pages.dim() == 3, "pages [n_pages, page_tokens, row]")
    return _cache_struct(pages, table)


def _cache_struct(pages, table):
    _need(table.dim() == 2 and table.dtype == _the_torch().int32 and (table.shape[1] == 1 or table.stride(1) == 1)
          and table.device == pages.device, "an int32 table [n_seqs, max_pages] on the pages' GPU")
    c = MoeLatentCache(pages.data_ptr(), table.data_ptr(),
                       table.stride(0) if table.shape[0] > 1 else table.shape[1], pages.shape[0], table.shape[0],
                       table.shape[1], 0)
    c.keep = (pages, table)
    return c


def _cache_of(spec, cache):
    """The cache's pages, as the description has them."""
    pages = cache.keep[0]
    if pages.dim() != 3 or pages.shape[1:] != (spec.page_tokens, spec.d_latent + spec.d_rope):
        raise ValueError("pages of %d tokens of %d" % (spec.page_tokens, spec.d_latent + spec.d_rope))
    return pages


def latent_append(spec, cache, kv, gamma, rope, seq, pos, status, q=None, q_out=None, stream=None):
    """moe_latent_append: ``kv`` fp32 ``[T, d_latent + d_rope]``, ``gamma`` fp16, ``rope`` fp32 ``[max_pos,
    d_rope / 2, 2]``, ``seq`` / ``pos`` int32 ``[T]``, ``q`` / ``q_out`` fp16 ``[T, H, d_nope + d_rope]``."""
    torch = _the_torch()
    T = kv.shape[0]
    _dense("pages, gamma", torch.float16, _cache_of(spec, cache), gamma)
    _dense("kv, rope", torch.float32, kv, rope)
    _dense("seq, pos, status", torch.int32, seq, pos, status)
    _need(kv.shape == (T, spec.d_latent + spec.d_rope) and rope.shape[1:] == (spec.d_rope // 2, 2)
          and rope.dim() == 3 and gamma.numel() == spec.d_latent and seq.numel() == T and pos.numel() == T,
          "kv [T, d_latent + d_rope], gamma [d_latent], rope [max_pos, d_rope / 2, 2], seq and pos [T]")
    _need((q is None) == (q_out is None), "q and q_out: both or none")
    if q is not None:
        _dense("q, q_out", torch.float16, q, q_out)
        _need(q.shape == q_out.shape == (T, spec.heads, spec.d_nope + spec.d_rope),
              "q and q_out [T, H, d_nope + d_rope]")
    _check(lib().moe_latent_append(ctypes.byref(spec), ctypes.byref(cache), _ptr(kv), _ptr(gamma), _ptr(rope),
                                   rope.shape[0], _ptr(seq), _ptr(pos), T, _ptr(q), _ptr(q_out), _ptr(status),
                                   _stream(stream)), "moe_latent_append")


def latent_decode_workspace_bytes(spec, B, max_len, prefix_len=0):
    return int(lib().moe_latent_decode_workspace_bytes(ctypes.byref(spec), B, max_len, prefix_len))


def _attends(spec, cache, w_kvb, q, out, workspace):
    _room(workspace)
    _dense("pages, w_kvb, q, out", _the_torch().float16, _cache_of(spec, cache), w_kvb, q, out)
    _need(w_kvb.shape == (spec.heads, spec.d_nope + spec.d_v, spec.d_latent)
          and q.shape[1:] == (spec.heads, spec.d_nope + spec.d_rope)
          and out.shape == (q.shape[0], spec.heads, spec.d_v),
          "w_kvb [H, d_nope + d_v, d_latent], q [T, H, d_nope + d_rope], out [T, H, d_v]")


def latent_decode(spec, cache, w_kvb, q, kv_len, max_len, out, status, workspace, prefix=None, prefix_len=0,
                  stream=None):
    """moe_latent_decode: ``q`` fp16 ``[B, H, d_nope + d_rope]``, ``kv_len`` int32 ``[B]``; ``prefix``: int32 page
    ids of ``prefix_len`` tokens that every sequence of the batch begins with. ``cache`` and ``kv_len`` are of the
    tokens behind the prefix: where table rows hold the prefix's k whole pages too, as those of forks do, a cache of
    the view ``table[:, k:]``."""
    torch = _the_torch()
    B = q.shape[0]
    _attends(spec, cache, w_kvb, q, out, workspace)
    _dense("kv_len, status", torch.int32, kv_len, status)
    _need(kv_len.numel() == B, "kv_len [B]")
    if prefix_len:
        _need(prefix is not None and prefix.numel() * spec.page_tokens >= prefix_len, "the prefix's page ids")
        _dense("prefix", torch.int32, prefix)
    _check(lib().moe_latent_decode(ctypes.byref(spec), ctypes.byref(cache), _ptr(w_kvb), _ptr(q), B, _ptr(kv_len),
                                   max_len, _ptr(prefix), prefix_len, _ptr(out), _ptr(status), _ptr(workspace),
                                   workspace.nbytes, _stream(stream)), "moe_latent_decode")


def latent_prefill_workspace_bytes(spec, B, kv_total):
    return int(lib().moe_latent_prefill_workspace_bytes(ctypes.byref(spec), B, kv_total))


def latent_prefill(spec, cache, w_kvb, q, q_start, kv_start, kv_total, max_q, out, status, workspace, stream=None):
    """moe_latent_prefill: ``q`` fp16 ``[T, H, d_nope + d_rope]``, ``q_start`` / ``kv_start`` int32 ``[B + 1]``."""
    torch = _the_torch()
    _attends(spec, cache, w_kvb, q, out, workspace)
    _dense("q_start, kv_start, status", torch.int32, q_start, kv_start, status)
    _need(q_start.numel() == kv_start.numel() >= 1, "q_start and kv_start [B + 1]")
    _check(lib().moe_latent_prefill(ctypes.byref(spec), ctypes.byref(cache), _ptr(w_kvb), _ptr(q), q.shape[0],
                                    _ptr(q_start), _ptr(kv_start), q_start.numel() - 1, kv_total, max_q, _ptr(out),
                                    _ptr(status), _ptr(workspace), workspace.nbytes, _stream(stream)),
           "moe_latent_prefill")


def latent4_page_bytes(spec):
    return int(lib().moe_latent4_page_bytes(ctypes.byref(spec)))


def latent4_cache(spec, pages, table):
    """moe_latent_cache of 4-bit ``pages`` uint8 ``[n_pages, latent4_page_bytes(spec)]`` and ``table`` int32 ``[n_seqs,
    max_pages]`` (rows may be strided), for the ``latent4_`` calls. The struct keeps both alive."""
    torch = _the_torch()
    _dense("pages", torch.uint8, pages)
    _need(pages.dim() == 2 and pages.shape[1] == latent4_page_bytes(spec), "uint8 pages [n_pages, %d]" % latent4_page_bytes(spec))
    return _cache_struct(pages, table)


def _cache4(spec, cache):
    pages = cache.keep[0]
    _dense("pages", _the_torch().uint8, pages)
    _need(pages.dim() == 2 and pages.shape[1] == latent4_page_bytes(spec), "a cache of latent4_cache with this description")


def latent4_append(spec, cache, kv, gamma, rope, seq, slot, pos, status, q=None, q_out=None, stream=None):
    """moe_latent4_append: as ``latent_append``, with each token's place ``slot`` int32 ``[T]`` beside its position."""
    torch = _the_torch()
    T = kv.shape[0]
    _cache4(spec, cache)
    _dense("gamma", torch.float16, gamma)
    _dense("kv, rope", torch.float32, kv, rope)
    _dense("seq, slot, pos, status", torch.int32, seq, slot, pos, status)
    _need(kv.shape == (T, spec.d_latent + spec.d_rope) and rope.shape[1:] == (spec.d_rope // 2, 2)
          and rope.dim() == 3 and gamma.numel() == spec.d_latent and seq.numel() == slot.numel() == pos.numel() == T,
          "kv [T, d_latent + d_rope], gamma [d_latent], rope [max_pos, d_rope / 2, 2], seq, slot and pos [T]")
    _need((q is None) == (q_out is None), "q and q_out: both or none")
    if q is not None:
        _dense("q, q_out", torch.float16, q, q_out)
        _need(q.shape == q_out.shape == (T, spec.heads, spec.d_nope + spec.d_rope),
              "q and q_out [T, H, d_nope + d_rope]")
    _check(lib().moe_latent4_append(ctypes.byref(spec), ctypes.byref(cache), _ptr(kv), _ptr(gamma), _ptr(rope),
                                    rope.shape[0], _ptr(seq), _ptr(slot), _ptr(pos), T, _ptr(q), _ptr(q_out),
                                    _ptr(status), _stream(stream)), "moe_latent4_append")


def latent4_read(spec, cache, seq, slot, rows, status, stream=None):
    """moe_latent4_read: the rows at ``seq`` / ``slot`` int32 ``[T]`` into ``rows`` fp16 ``[T, d_latent + d_rope]``."""
    torch = _the_torch()
    T = rows.shape[0]
    _cache4(spec, cache)
    _dense("rows", torch.float16, rows)
    _dense("seq, slot, status", torch.int32, seq, slot, status)
    _need(rows.shape == (T, spec.d_latent + spec.d_rope) and seq.numel() == slot.numel() == T,
          "rows [T, d_latent + d_rope], seq and slot [T]")
    _check(lib().moe_latent4_read(ctypes.byref(spec), ctypes.byref(cache), _ptr(seq), _ptr(slot), T, _ptr(rows),
                                  _ptr(status), _stream(stream)), "moe_latent4_read")


def _attends4(spec, cache, w_kvb, q, out, workspace, sums, B, least):
    """The checks that both forms share; the stride of the sums' rows."""
    torch = _the_torch()
    _room(workspace)
    _cache4(spec, cache)
    _dense("w_kvb, q, out", torch.float16, w_kvb, q, out)
    _need(w_kvb.shape == (spec.heads, spec.d_nope + spec.d_v, spec.d_latent)
          and q.shape[1:] == (spec.heads, spec.d_nope + spec.d_rope)
          and out.shape == (q.shape[0], spec.heads, spec.d_v),
          "w_kvb [H, d_nope + d_v, d_latent], q [T, H, d_nope + d_rope], out [T, H, d_v]")
    if sums is None:
        return 0
    _need(sums.dtype == torch.float32 and sums.dim() == 2 and sums.shape[0] >= B and sums.shape[1] >= least
          and (sums.shape[1] == 1 or sums.stride(1) == 1) and sums.get_device() == _current_device(),
          "sums: fp32 [B, at least %d] with unit column stride on the current GPU" % least)
    return sums.stride(0) if sums.shape[0] > 1 else sums.shape[1]


def latent4_decode_workspace_bytes(spec, B, max_len, sums=False):
    return int(lib().moe_latent4_decode_workspace_bytes(ctypes.byref(spec), B, max_len, int(sums)))


def latent4_decode(spec, cache, w_kvb, q, kv_len, max_len, out, status, workspace, sums=None, stream=None):
    """moe_latent4_decode: as ``latent_decode``; ``sums`` fp32 ``[B, >= max_len]`` or None, to which each token's weights
    over all heads are added."""
    B = q.shape[0]
    stride = _attends4(spec, cache, w_kvb, q, out, workspace, sums, B, max_len)
    _dense("kv_len, status", _the_torch().int32, kv_len, status)
    _need(kv_len.numel() == B, "kv_len [B]")
    _check(lib().moe_latent4_decode(ctypes.byref(spec), ctypes.byref(cache), _ptr(w_kvb), _ptr(q), B, _ptr(kv_len),
                                    max_len, _ptr(out), _ptr(sums), stride, _ptr(status), _ptr(workspace),
                                    workspace.nbytes, _stream(stream)), "moe_latent4_decode")


def latent4_prefill_workspace_bytes(spec, T, B, kv_total, sums=False):
    return int(lib().moe_latent4_prefill_workspace_bytes(ctypes.byref(spec), T, B, kv_total, int(sums)))


def latent4_prefill(spec, cache, w_kvb, q, q_start, kv_start, kv_total, max_q, out, status, workspace, sums=None,
                    stream=None):
    """moe_latent4_prefill: as ``latent_prefill``; ``sums`` fp32 ``[B, tokens]`` or None (tokens beyond it get none)."""
    B = q_start.numel() - 1
    stride = _attends4(spec, cache, w_kvb, q, out, workspace, sums, B, 1)
    _dense("q_start, kv_start, status", _the_torch().int32, q_start, kv_start, status)
    _need(q_start.numel() == kv_start.numel() >= 1, "q_start and kv_start [B + 1]")
    _check(lib().moe_latent4_prefill(ctypes.byref(spec), ctypes.byref(cache), _ptr(w_kvb), _ptr(q), q.shape[0],
                                     _ptr(q_start), _ptr(kv_start), B, kv_total, max_q, _ptr(out), _ptr(sums), stride,
                                     0 if sums is None else sums.shape[1], _ptr(status), _ptr(workspace),
                                     workspace.nbytes, _stream(stream)), "moe_latent4_prefill")


def evict_select(sums, kv_len, budget, sinks, recent, keep, sums_out, status, stream=None):
    """moe_evict_select: ``sums`` fp32 ``[layers, B, width]``, ``kv_len`` int32 ``[B]``, ``keep`` int32 ``[layers, B,
    budget]``; ``sums_out`` may be ``sums``."""
    torch = _the_torch()
    _dense("sums, sums_out", torch.float32, sums, sums_out)
    _dense("kv_len, keep, status", torch.int32, kv_len, keep, status)
    _need(sums.dim() == 3 and sums_out.shape == sums.shape and kv_len.numel() == sums.shape[1]
          and keep.shape == (sums.shape[0], sums.shape[1], budget),
          "sums and sums_out [layers, B, width], kv_len [B], keep [layers, B, budget]")
    _check(lib().moe_evict_select(_ptr(sums), _ptr(sums_out), sums.shape[0], sums.shape[1], sums.shape[2], _ptr(kv_len),
                                  budget, sinks, recent, _ptr(keep), _ptr(status), _stream(stream)), "moe_evict_select")


def latent4_move(spec, pages, table, keep, to_table, status, stream=None):
    """moe_latent4_move on 4-bit ``pages`` uint8 ``[layers, n_pages, page bytes]`` (a layer contiguous, layers may be
    strided): the rows ``keep`` int32 ``[layers, B, budget]`` of the sequences of ``table`` go to the pages ``to_table``
    int32 ``[B, >= ceil(budget / page_tokens)]``."""
    torch = _the_torch()
    _need(pages.dim() == 3 and keep.dim() == 3 and pages.shape[0] == keep.shape[0] > 0 and to_table.dim() == 2
          and to_table.shape[0] == keep.shape[1], "pages [layers, n_pages, bytes], keep [layers, B, budget], to_table [B, pages]")
    cache = latent4_cache(spec, pages[0], table)
    need = -(-keep.shape[2] // spec.page_tokens)
    _need(to_table.shape[1] >= need, "to_table: %d pages a sequence" % need)
    _dense("keep, to_table, status", torch.int32, keep, to_table, status)
    _check(lib().moe_latent4_move(ctypes.byref(spec), ctypes.byref(cache), pages.shape[0], pages.stride(0), _ptr(keep),
                                  keep.shape[1], keep.shape[2], _ptr(to_table), to_table.shape[1], _ptr(status),
                                  _stream(stream)), "moe_latent4_move")


class PagePool:
    """The library's page bookkeeping (host only): reference counts, forks, compaction."""

    def __init__(self, n_pages, page_tokens):
        h = c_void_p()
        _check(lib().moe_page_pool_create(n_pages, page_tokens, ctypes.byref(h)), "moe_page_pool_create")
        self.handle, self.n_pages, self.page_tokens = h, n_pages, page_tokens

    def available(self):
        return _check(lib().moe_page_pool_available(self.handle), "moe_page_pool_available")

    def refs(self, page):
        return _check(lib().moe_page_pool_refs(self.handle, page), "moe_page_pool_refs")

    def alloc(self, n):
        out = np.zeros(max(n, 1), dtype=np.int32)
        _check(lib().moe_page_pool_alloc(self.handle, n, out.ctypes.data), "moe_page_pool_alloc")
        return out[:n].tolist()

    def fork(self, pages, n_tokens):
        """(pages of the fork, the (from, to) pairs to copy)."""
        p = _i32(pages)
        n = -(-n_tokens // self.page_tokens)
        _need(n <= len(p), "%d tokens need %d pages" % (n_tokens, n))
        out, copy = np.zeros(max(n, 1), dtype=np.int32), np.zeros(2, dtype=np.int32)
        k = _check(lib().moe_page_pool_fork(self.handle, p.ctypes.data, n_tokens, out.ctypes.data, copy.ctypes.data),
                   "moe_page_pool_fork")
        return out[:n].tolist(), [tuple(copy.tolist())] if k else []

    def free(self, pages):
        p = _i32(pages)
        _check(lib().moe_page_pool_free(self.handle, p.ctypes.data, len(p)), "moe_page_pool_free")

    def compact(self):
        """(int32 [n, 2] moves, int32 [n_pages] remap)."""
        moves, remap = np.zeros((self.n_pages, 2), dtype=np.int32), np.zeros(self.n_pages, dtype=np.int32)
        n = _check(lib().moe_page_pool_compact(self.handle, moves.ctypes.data, remap.ctypes.data),
                   "moe_page_pool_compact")
        return moves[:n], remap

    def close(self):
        if self.handle:
            lib().moe_page_pool_destroy(self.handle)
            self.handle = None

    def __del__(self, _finalizing=sys.is_finalizing):
        # no runtime calls while the interpreter shuts down: close() explicitly
        if _finalizing():
            return
        try:
            self.close()
        except Exception:
            pass


def page_copy(pages, pairs, status, stream=None):
    """moe_page_copy on ``pages [n_layers, n_pages, ...]`` (pages contiguous, layers may be strided); ``pairs``
    int32 ``[n, 2]`` on the GPU."""
    torch = _the_torch()
    _need(pages.dim() >= 3 and pages.shape[0] > 0 and pairs.dim() == 2 and pairs.shape[1] == 2,
          "pages [n_layers, n_pages, ...], pairs [n, 2]")
    _dense("pages of a layer", pages.dtype, pages if pages.is_contiguous() else pages[0])
    _dense("pairs, status", torch.int32, pairs, status)
    size = pages.element_size()
    _check(lib().moe_page_copy(_ptr(pages), pages.shape[0], pages.stride(0) * size, pages.stride(1) * size,
                               pages.shape[1], _ptr(pairs), pairs.shape[0], _ptr(status), _stream(stream)),
           "moe_page_copy")


def page_remap(table, remap, table_out, status, stream=None):
    """moe_page_remap: int32 tensors; ``table_out`` may be ``table``."""
    torch = _the_torch()
    _dense("table, remap, table_out, status", torch.int32, table, remap, table_out, status)
    _need(table_out.numel() == table.numel(), "tables of one size")
    _check(lib().moe_page_remap(_ptr(table), table.numel(), _ptr(remap), remap.numel(), _ptr(table_out), _ptr(status),
                                _stream(stream)), "moe_page_remap")
