"""ctypes binding of include/rpo.h: same names, argument marshalling only.

Device buffers are torch CUDA tensors (their data pointers are passed through); every
step of the path runs inside the library's kernels.
"""
import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None

EXPORTED_SYMBOLS = [
    "rpo_strerror", "rpo_shape_preset", "rpo_create", "rpo_destroy", "rpo_init_weights", "rpo_read_tensor",
    "rpo_write_tensor", "rpo_prefill_prefix", "rpo_decode_suffix", "rpo_decode_wave", "rpo_token_logprobs", "rpo_release_groups",
    "rpo_policy_objective", "rpo_rollout_host", "rpo_sample_rows", "rpo_sample_rows_noalloc", "rpo_gemm", "rpo_gemm_bench", "rpo_chunk_attention", "rpo_attention_mass", "rpo_evict_cache", "rpo_tree_attention", "rpo_verify_drafts",
    "rpo_commit_path", "rpo_fork_pages", "rpo_reserve_pages", "rpo_device_status", "rpo_debug_tap", "rpo_counters", "rpo_set_option", "rpo_profile_read",
]


class RpoError(RuntimeError):
    def __init__(self, code, what):
        super().__init__(f"{what}: {code} ({load_library().rpo_strerror(code).decode()})")
        self.code = code


class Shape(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("d_ffn", C.c_int32), ("vocab", C.c_int32), ("rope_base", C.c_float),
                ("rms_eps", C.c_float), ("dtype", C.c_int32), ("kv_block_tokens", C.c_int32)]


class Limits(C.Structure):
    _fields_ = [("kv_pool_blocks", C.c_int64), ("max_groups", C.c_int32), ("max_seqs", C.c_int32),
                ("max_chunk_tokens", C.c_int32), ("max_positions", C.c_int32)]


class Sampler(C.Structure):
    _fields_ = [("temperature", C.c_float), ("top_p", C.c_float), ("greedy", C.c_int32), ("eos_id", C.c_int32),
                ("seed", C.c_uint64)]

    def __init__(self, temperature=1.0, top_p=1.0, greedy=False, eos_id=-1, seed=0):
        super().__init__(float(temperature), float(top_p), int(bool(greedy)), int(eos_id), int(seed))


class ObjectiveCfg(C.Structure):
    _fields_ = [("clip_eps", C.c_float), ("beta", C.c_float), ("alpha", C.c_float), ("reward_min", C.c_float),
                ("reward_max", C.c_float), ("length_shaping", C.c_int32)]

    def __init__(self, clip_eps=0.2, beta=0.0, alpha=0.01, reward_min=0.5, reward_max=1.0, length_shaping=True):
        super().__init__(float(clip_eps), float(beta), float(alpha), float(reward_min), float(reward_max), int(bool(length_shaping)))


class Group(C.Structure):
    _fields_ = [("group_id", C.c_int32), ("prefix_len", C.c_int32), ("slot", C.c_int32), ("n_blocks", C.c_int32)]


class _PagedKVStruct(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("d_block_table", C.c_void_p), ("d_lens", C.c_void_p), ("n_blocks", C.c_int32),
                ("n_seqs", C.c_int32), ("table_stride", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32)]


class _ChunkCfg(C.Structure):
    _fields_ = [("scale", C.c_float), ("window", C.c_int32), ("sinks", C.c_int32)]


class PagedKV:
    """rpo_paged_kv: one layer's paged K/V cache in tensors of the caller.

    d_k, d_v [n_kv_heads, n_blocks, 16, head_dim] (float32 or bfloat16), d_block_table int32 [n_seqs, table_stride],
    d_lens int32 [n_seqs].  Keeps references to the tensors; build it once and reuse it."""

    def __init__(self, d_k, d_v, d_block_table, d_lens):
        if (d_k.dim() != 4 or d_k.shape[2] != 16 or d_v.shape != d_k.shape or d_v.dtype != d_k.dtype or not d_k.is_contiguous()
                or not d_v.is_contiguous() or d_v.device != d_k.device):
            raise ValueError("d_k and d_v must be contiguous [n_kv_heads, n_blocks, 16, head_dim] of one type on one device")
        self.device = d_k.device
        _expect(d_block_table, "d_block_table", "int32", (d_lens.shape[0], d_block_table.shape[-1]), self.device)
        _expect(d_lens, "d_lens", "int32", (d_block_table.shape[0],), self.device)
        self.d_k, self.d_v, self.d_block_table, self.d_lens = d_k, d_v, d_block_table, d_lens
        self.dtype = d_k.dtype
        hkv, n_blocks, _, dh = d_k.shape
        self.struct = _PagedKVStruct(_ptr(d_k), _ptr(d_v), _ptr(d_block_table), _ptr(d_lens), n_blocks, d_block_table.shape[0],
                                     d_block_table.shape[1], hkv, dh)
        self.ref = C.byref(self.struct)


class PagedLayers:
    """The caches of all layers of a model (PagedKV objects that share their block table and lengths): what calls that move rows
    or pages work on.  Keeps references; build it once and reuse it."""

    def __init__(self, layers):
        self.layers = list(layers)
        if not self.layers:
            raise ValueError("at least one layer is needed")
        first = self.layers[0]
        for kv in self.layers:
            if (kv.dtype is not first.dtype or kv.device != first.device or kv.d_k.shape != first.d_k.shape
                    or kv.d_block_table.data_ptr() != first.d_block_table.data_ptr() or kv.d_block_table.shape != first.d_block_table.shape
                    or kv.d_lens.data_ptr() != first.d_lens.data_ptr()):
                raise ValueError("the layers must have one type, device and shape, and share d_block_table and d_lens")
        self.dtype, self.device, self.n_seqs = first.dtype, first.device, first.struct.n_seqs
        self.array = (_PagedKVStruct * len(self.layers))(*[kv.struct for kv in self.layers])


class _PagePoolStruct(C.Structure):
    _fields_ = [("d_refs", C.c_void_p), ("d_free", C.c_void_p), ("d_n_free", C.c_void_p), ("d_block_table", C.c_void_p), ("d_held", C.c_void_p),
                ("n_blocks", C.c_int32), ("n_seqs", C.c_int32), ("table_stride", C.c_int32)]


class PagePool:
    """rpo_page_pool: reference counts and free pages in int32 tensors of the caller.

    d_refs, d_free [n_blocks], d_n_free [1], d_block_table [n_seqs, table_stride] (the caches'), d_held [n_seqs]."""

    def __init__(self, d_refs, d_free, d_n_free, d_block_table, d_held):
        self.device = d_block_table.device
        for t, name, shape in ((d_refs, "d_refs", d_free.shape[:1]), (d_free, "d_free", d_refs.shape[:1]), (d_n_free, "d_n_free", (1,)),
                               (d_block_table, "d_block_table", (d_held.shape[0], d_block_table.shape[-1])), (d_held, "d_held", (d_block_table.shape[0],))):
            _expect(t, name, "int32", shape, self.device)
        self.d_refs, self.d_free, self.d_n_free, self.d_block_table, self.d_held = d_refs, d_free, d_n_free, d_block_table, d_held
        self.struct = _PagePoolStruct(_ptr(d_refs), _ptr(d_free), _ptr(d_n_free), _ptr(d_block_table), _ptr(d_held), d_refs.shape[0],
                                      d_block_table.shape[0], d_block_table.shape[1])
        self.ref = C.byref(self.struct)

    @classmethod
    def empty(cls, n_blocks, n_seqs, table_stride, device="cuda"):
        """A pool of free pages (page 0 on top of the stack), with a table of sequences that hold none."""
        import torch
        i32 = dict(dtype=torch.int32, device=device)
        return cls(torch.zeros(n_blocks, **i32), torch.arange(n_blocks - 1, -1, -1, **i32), torch.full((1,), n_blocks, **i32),
                   torch.full((n_seqs, table_stride), -1, **i32), torch.zeros(n_seqs, **i32))


def load_library(path=None):
    """Load librpo.so (building it first if it is missing) and declare the prototypes."""
    global _LIB
    if _LIB is not None and path is None:
        return _LIB
    path = path or os.path.join(_HERE, "librpo.so")
    if not os.path.exists(path):
        from . import build as _build
        _build.build()
    lib = C.CDLL(path)
    vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
    lib.rpo_strerror.restype = C.c_char_p; lib.rpo_strerror.argtypes = [C.c_int]
    lib.rpo_shape_preset.argtypes = [C.c_char_p, C.POINTER(Shape)]
    lib.rpo_create.argtypes = [C.POINTER(vp), C.POINTER(Shape), C.POINTER(Limits), vp]
    lib.rpo_destroy.argtypes = [vp]
    lib.rpo_init_weights.argtypes = [vp, C.c_uint64, f32]
    lib.rpo_read_tensor.argtypes = [vp, C.c_char_p, vp, C.c_size_t]
    lib.rpo_write_tensor.argtypes = [vp, C.c_char_p, vp, C.c_size_t]
    lib.rpo_prefill_prefix.argtypes = [vp, i32, vp, vp, vp, C.POINTER(Group)]
    lib.rpo_decode_suffix.argtypes = [vp, i32, C.POINTER(Group), i32, i32, C.POINTER(Sampler), vp, vp, vp, vp, vp]
    lib.rpo_decode_wave.argtypes = [vp, i32, C.POINTER(Group), i32, i32, i32, C.POINTER(Sampler), vp, vp, vp, vp]
    lib.rpo_token_logprobs.argtypes = [vp, i32, C.POINTER(Group), i32, i32, vp, vp, f32, vp, vp]
    lib.rpo_policy_objective.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, C.POINTER(ObjectiveCfg), vp, vp, vp, vp, vp]
    lib.rpo_release_groups.argtypes = [vp, i32, C.POINTER(Group)]
    lib.rpo_rollout_host.argtypes = [vp, i32, vp, vp, vp, i32, i32, C.POINTER(Sampler), vp, vp, vp, i32, vp]
    lib.rpo_sample_rows.argtypes = [vp, i32, i32, vp, C.POINTER(Sampler), vp, i32, vp, vp]
    lib.rpo_sample_rows_noalloc.argtypes = [i32, i32, vp, C.POINTER(Sampler), vp, i32, vp, vp, vp]
    lib.rpo_gemm.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp]
    lib.rpo_gemm_bench.argtypes = [vp, i32, i32, i32, vp, C.POINTER(vp), i32, i32, C.POINTER(f32)]
    pkv, ccfg = C.POINTER(_PagedKVStruct), C.POINTER(_ChunkCfg)
    lib.rpo_chunk_attention.argtypes = [vp, pkv, i32, i32, i32, vp, i64, vp, vp, i64, vp, ccfg, vp, vp]
    lib.rpo_attention_mass.argtypes = [vp, pkv, i32, i32, i32, vp, i64, vp, ccfg, vp, vp, vp, i32]
    lib.rpo_evict_cache.argtypes = [vp, pkv, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, i32]
    lib.rpo_tree_attention.argtypes = [vp, pkv, i32, i32, i32, vp, i64, vp, vp, i64, vp, vp, ccfg, vp, vp]
    lib.rpo_verify_drafts.argtypes = [vp, i32, i32, i32, vp, i64, vp, i64, vp, vp, vp, vp, C.POINTER(Sampler), i32, vp, vp, vp, vp]
    pool = C.POINTER(_PagePoolStruct)
    lib.rpo_commit_path.argtypes = [vp, pkv, i32, vp, vp, i32, vp, vp]
    lib.rpo_fork_pages.argtypes = [vp, pool, pkv, i32, i32, vp, vp, vp, vp]
    lib.rpo_reserve_pages.argtypes = [vp, pool, pkv, i32, vp, vp]
    lib.rpo_device_status.argtypes = [vp, C.POINTER(i32)]
    lib.rpo_debug_tap.argtypes = [vp, vp, i64, C.POINTER(i64)]
    lib.rpo_counters.argtypes = [vp, C.POINTER(i64), C.POINTER(i64)]
    lib.rpo_set_option.argtypes = [vp, C.c_char_p, i32]
    lib.rpo_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(i64), i32]
    for name in EXPORTED_SYMBOLS:
        if name != "rpo_strerror":
            getattr(lib, name).restype = C.c_int
    if path == os.path.join(_HERE, "librpo.so"):
        _LIB = lib
    return lib


def shape_preset(name, **overrides):
    s = Shape()
    rc = load_library().rpo_shape_preset(name.encode(), C.byref(s))
    if rc != 0:
        raise RpoError(rc, f"rpo_shape_preset({name})")
    for k, v in overrides.items():
        setattr(s, k, v)
    return s


def shape_from_dict(d):
    s = Shape()
    for k in ("n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab"):
        setattr(s, k, int(d[k]))
    s.rope_base = float(d.get("rope_base", 10000.0)); s.rms_eps = float(d.get("rms_eps", 1e-6))
    s.dtype = 1 if d.get("dtype", "fp32") == "bf16" else 0
    s.kv_block_tokens = 16
    return s


def _ptr(t):
    """Device/host pointer of a torch tensor or numpy array (None -> NULL)."""
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        assert t.flags["C_CONTIGUOUS"]
        return t.ctypes.data
    assert t.is_contiguous()
    return t.data_ptr()


_DTYPES = {}


def _dtype(name):
    """torch.<name>, looked up once (torch is imported with the first tensor, not with this module)."""
    if name not in _DTYPES:
        import torch
        _DTYPES[name] = getattr(torch, name)
    return _DTYPES[name]


def _expect(t, name, dtype, shape, device):
    """Refuse a tensor of another type, shape, layout or device than a call takes."""
    if t.dtype is not _dtype(dtype) or t.shape != shape or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")


def _head_rows(t, name, dtype, heads, dh, device, n_rows=None):
    """Elements between the rows of a [rows, heads, head_dim] view whose rows are contiguous (a slice of a fused projection is)."""
    shape = t.shape
    if len(shape) != 3 or t.dtype is not dtype or shape[1] != heads or shape[2] != dh or (n_rows is not None and shape[0] != n_rows):
        raise ValueError(f"{name} must be {dtype} [{'rows' if n_rows is None else n_rows}, {heads}, {dh}], got {t.dtype} {tuple(shape)}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the cache on {device}")
    stride = t.stride()
    if shape[0] and (stride[2] != 1 or (heads > 1 and stride[1] != dh)):      # (strides of nothing may be anything)
        raise ValueError(f"{name}: the heads of a row must be contiguous")
    return stride[0] if shape[0] > 1 else heads * dh


def _check(rc, what):
    if rc != 0:
        raise RpoError(rc, what)


def sample_rows_noalloc(d_logits, sampler, d_seq_ids, step, d_tokens_out, d_logprobs_out=None, stream=None):
    """rpo_sample_rows_noalloc: the sampler on caller-supplied logits [n_rows, vocab] without a context
    and without any allocation (its scratch is a fixed 16 MiB array inside the library, so
    n_rows * vocab is limited to 4 Mi words).  `stream` is a torch.cuda.Stream or None."""
    n, v = d_logits.shape
    stream_ptr = None if stream is None else C.c_void_p(stream.cuda_stream)
    _check(load_library().rpo_sample_rows_noalloc(n, v, _ptr(d_logits), C.byref(sampler), _ptr(d_seq_ids), int(step),
                                                  _ptr(d_tokens_out), _ptr(d_logprobs_out), stream_ptr),
           "rpo_sample_rows_noalloc")


class Context:
    """Owns one rpo_ctx.  Methods mirror the C calls one to one."""

    device = None                       # of the context's memory

    def __init__(self, shape, kv_pool_blocks, max_groups, max_seqs, max_chunk_tokens, max_positions, stream=None):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("paper_2601_19404_b200 needs a CUDA device: the library has no CPU path")
        self.lib = load_library()
        self.shape = shape if isinstance(shape, Shape) else shape_from_dict(shape)
        self.limits = Limits(int(kv_pool_blocks), int(max_groups), int(max_seqs), int(max_chunk_tokens), int(max_positions))
        self.handle = C.c_void_p()
        stream_ptr = None if stream is None else C.c_void_p(stream.cuda_stream)
        _check(self.lib.rpo_create(C.byref(self.handle), C.byref(self.shape), C.byref(self.limits), stream_ptr), "rpo_create")
        self.device = torch.device("cuda", torch.cuda.current_device())

    def close(self):
        h = getattr(self, "handle", None)
        if h is not None and h.value:
            self.lib.rpo_destroy(h)
            h.value = None

    __del__ = close

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    @property
    def storage_dtype(self):
        return np.uint16 if self.shape.dtype == 1 else np.float32

    def init_weights(self, seed=0, std=0.02):
        _check(self.lib.rpo_init_weights(self.handle, int(seed), float(std)), "rpo_init_weights")

    def tensor_shape(self, name):
        s = self.shape
        qo, kvo = s.n_q_heads * s.head_dim, s.n_kv_heads * s.head_dim
        leaf = name.split(".")[-1]
        table = {"embed": (s.vocab, s.d_model), "lm_head": (s.vocab, s.d_model), "gf": (s.d_model,),
                 "wq": (qo, s.d_model), "wk": (kvo, s.d_model), "wv": (kvo, s.d_model), "wo": (s.d_model, qo),
                 "wg": (s.d_ffn, s.d_model), "wu": (s.d_ffn, s.d_model), "wd": (s.d_model, s.d_ffn),
                 "g1": (s.d_model,), "g2": (s.d_model,)}
        return table[leaf]

    def read_tensor(self, name):
        gain = name.split(".")[-1] in ("gf", "g1", "g2")
        out = np.empty(self.tensor_shape(name), dtype=np.float32 if gain else self.storage_dtype)
        _check(self.lib.rpo_read_tensor(self.handle, name.encode(), out.ctypes.data, out.nbytes), f"rpo_read_tensor({name})")
        return out

    def write_tensor(self, name, array):
        gain = name.split(".")[-1] in ("gf", "g1", "g2")
        a = np.ascontiguousarray(array, dtype=np.float32 if gain else self.storage_dtype)
        assert a.shape == tuple(self.tensor_shape(name))
        _check(self.lib.rpo_write_tensor(self.handle, name.encode(), a.ctypes.data, a.nbytes), f"rpo_write_tensor({name})")

    def prefill_prefix(self, d_tokens, h_offsets, group_ids=None):
        n = len(h_offsets) - 1
        off = np.ascontiguousarray(h_offsets, dtype=np.int32)
        ids = None if group_ids is None else np.ascontiguousarray(group_ids, dtype=np.int32)
        groups = (Group * n)()
        _check(self.lib.rpo_prefill_prefix(self.handle, n, _ptr(d_tokens), off.ctypes.data,
                                           None if ids is None else ids.ctypes.data, groups), "rpo_prefill_prefix")
        return groups

    def decode_suffix(self, groups, G, max_new, sampler, d_tokens_out, d_lens_out, d_logprobs_out=None,
                      d_forced_tokens=None, d_logits_dbg=None):
        _check(self.lib.rpo_decode_suffix(self.handle, len(groups), groups, int(G), int(max_new), C.byref(sampler),
                                          _ptr(d_forced_tokens), _ptr(d_tokens_out), _ptr(d_lens_out),
                                          _ptr(d_logprobs_out), _ptr(d_logits_dbg)), "rpo_decode_suffix")

    def decode_wave(self, groups, G, max_new, max_total, sampler, d_tokens_out, d_lens_out, d_logprobs_out=None,
                    d_forced_tokens=None):
        _check(self.lib.rpo_decode_wave(self.handle, len(groups), groups, int(G), int(max_new), int(max_total),
                                        C.byref(sampler), _ptr(d_forced_tokens), _ptr(d_tokens_out), _ptr(d_lens_out),
                                        _ptr(d_logprobs_out)), "rpo_decode_wave")

    def token_logprobs(self, groups, G, max_new, d_tokens, d_lens, d_logprobs_out, inv_temperature=1.0, d_logits_dbg=None):
        _check(self.lib.rpo_token_logprobs(self.handle, len(groups), groups, int(G), int(max_new), _ptr(d_tokens),
                                           _ptr(d_lens), float(inv_temperature), _ptr(d_logprobs_out),
                                           _ptr(d_logits_dbg)), "rpo_token_logprobs")

    def policy_objective(self, n_groups, G, max_new, d_logp_new, d_logp_old, d_lens, d_raw_rewards, cfg, d_rewards_out,
                         d_advantages_out, d_group_objective_out, d_objective_out, d_logp_ref=None, d_resp_lens=None,
                         d_token_loss_out=None):
        _check(self.lib.rpo_policy_objective(self.handle, int(n_groups), int(G), int(max_new), _ptr(d_logp_new), _ptr(d_logp_old),
                                             _ptr(d_logp_ref), _ptr(d_lens), _ptr(d_resp_lens), _ptr(d_raw_rewards), C.byref(cfg),
                                             _ptr(d_rewards_out), _ptr(d_advantages_out), _ptr(d_token_loss_out),
                                             _ptr(d_group_objective_out), _ptr(d_objective_out)), "rpo_policy_objective")

    def release_groups(self, groups):
        _check(self.lib.rpo_release_groups(self.handle, len(groups), groups), "rpo_release_groups")

    def rollout_host(self, h_tokens, h_offsets, G, max_new, sampler, h_tokens_out, h_lens_out, h_logprobs_out=None,
                     h_policy_logprobs_out=None, group_ids=None):
        n = len(h_offsets) - 1
        off = np.ascontiguousarray(h_offsets, dtype=np.int32)
        ids = None if group_ids is None else np.ascontiguousarray(group_ids, dtype=np.int32)
        _check(self.lib.rpo_rollout_host(self.handle, n, _ptr(h_tokens), off.ctypes.data,
                                         None if ids is None else ids.ctypes.data, int(G), int(max_new),
                                         C.byref(sampler), _ptr(h_tokens_out), _ptr(h_lens_out), _ptr(h_logprobs_out),
                                         int(h_policy_logprobs_out is not None), _ptr(h_policy_logprobs_out)),
               "rpo_rollout_host")

    def sample_rows(self, d_logits, sampler, d_seq_ids, step, d_tokens_out, d_logprobs_out=None):
        n, v = d_logits.shape
        _check(self.lib.rpo_sample_rows(self.handle, n, v, _ptr(d_logits), C.byref(sampler), _ptr(d_seq_ids), int(step),
                                        _ptr(d_tokens_out), _ptr(d_logprobs_out)), "rpo_sample_rows")

    def gemm(self, d_A, d_W, d_C, impl=0):
        M, K = d_A.shape
        N = d_W.shape[0]
        _check(self.lib.rpo_gemm(self.handle, int(impl), M, N, K, _ptr(d_A), _ptr(d_W), _ptr(d_C)), "rpo_gemm")

    def gemm_bench(self, d_A, d_W_list, iters):
        """Mean device milliseconds per launch of the tensor-core GEMM A W^T, cycling through d_W_list."""
        M, K = d_A.shape
        N = d_W_list[0].shape[0]
        ptrs = (C.c_void_p * len(d_W_list))(*[w.data_ptr() for w in d_W_list])
        ms = C.c_float()
        _check(self.lib.rpo_gemm_bench(self.handle, M, N, K, _ptr(d_A), ptrs, len(d_W_list), int(iters), C.byref(ms)),
               "rpo_gemm_bench")
        return ms.value

    def _paged_dtype(self, kv):
        if kv.dtype is not _dtype("bfloat16" if self.shape.dtype == 1 else "float32"):
            raise ValueError(f"a cache of {kv.dtype} needs a context of that storage type")
        if self.device is not None and kv.device != self.device:
            raise ValueError(f"the cache is on {kv.device}, the context on {self.device}")
        return kv.dtype

    def _chunk_cfg(self, kv, scale, window, sinks):
        return _ChunkCfg(kv.struct.head_dim ** -0.5 if scale is None else scale, window, sinks)

    def _chunk_rows(self, d_q, kv, d_q_offsets, d_out, d_lse_out, d_k_new, d_v_new):
        """Checks what attention calls share; (rows, query heads, row strides of d_q and of d_k_new)."""
        dt, st = self._paged_dtype(kv), kv.struct
        n, hq = d_q.shape[0], d_q.shape[1]
        q_stride = _head_rows(d_q, "d_q", dt, hq, st.head_dim, kv.device)
        new_stride = 0
        if (d_k_new is None) != (d_v_new is None):
            raise ValueError("d_k_new and d_v_new go together")
        if d_k_new is not None:
            new_stride = _head_rows(d_k_new, "d_k_new", dt, st.n_kv_heads, st.head_dim, kv.device, n)
            if _head_rows(d_v_new, "d_v_new", dt, st.n_kv_heads, st.head_dim, kv.device, n) != new_stride:
                raise ValueError("d_k_new and d_v_new must have the same row stride")
        _expect(d_q_offsets, "d_q_offsets", "int32", (st.n_seqs + 1,), kv.device)
        if d_out.dtype is not dt or d_out.shape != d_q.shape or not d_out.is_contiguous() or d_out.device != kv.device:
            raise ValueError("d_out must be contiguous, of d_q's type and shape, on its device")
        if d_lse_out is not None:
            _expect(d_lse_out, "d_lse_out", "float32", (n, hq), kv.device)
        return n, hq, q_stride, new_stride

    def chunk_attention(self, d_q, kv, d_q_offsets, max_chunk, d_out, d_lse_out=None, d_k_new=None, d_v_new=None, scale=None, window=0, sinks=0):
        """rpo_chunk_attention: d_q [rows, n_q_heads, head_dim] (rows may be strided), kv a PagedKV, d_out contiguous, d_lse_out
        float32 [rows, n_q_heads].  scale defaults to head_dim ** -0.5."""
        n, hq, q_stride, new_stride = self._chunk_rows(d_q, kv, d_q_offsets, d_out, d_lse_out, d_k_new, d_v_new)
        cfg = self._chunk_cfg(kv, scale, window, sinks)
        _check(self.lib.rpo_chunk_attention(self.handle, kv.ref, n, hq, max_chunk, d_q.data_ptr(), q_stride,
                                            None if d_k_new is None else d_k_new.data_ptr(), None if d_v_new is None else d_v_new.data_ptr(),
                                            new_stride, d_q_offsets.data_ptr(), C.byref(cfg), d_out.data_ptr(),
                                            None if d_lse_out is None else d_lse_out.data_ptr()), "rpo_chunk_attention")

    def tree_attention(self, d_q, kv, d_q_offsets, d_parents, max_nodes, d_out, d_lse_out=None, d_k_new=None, d_v_new=None, scale=None, window=0,
                       sinks=0):
        """rpo_tree_attention: as chunk_attention, the rows of a sequence being the nodes of a tree; d_parents int32 [rows], -1 a child of
        the last cached token, -2 no node."""
        n, hq, q_stride, new_stride = self._chunk_rows(d_q, kv, d_q_offsets, d_out, d_lse_out, d_k_new, d_v_new)
        _expect(d_parents, "d_parents", "int32", (n,), kv.device)
        cfg = self._chunk_cfg(kv, scale, window, sinks)
        _check(self.lib.rpo_tree_attention(self.handle, kv.ref, n, hq, max_nodes, d_q.data_ptr(), q_stride,
                                           None if d_k_new is None else d_k_new.data_ptr(), None if d_v_new is None else d_v_new.data_ptr(),
                                           new_stride, d_q_offsets.data_ptr(), d_parents.data_ptr(), C.byref(cfg), d_out.data_ptr(),
                                           None if d_lse_out is None else d_lse_out.data_ptr()), "rpo_tree_attention")

    def verify_drafts(self, d_logits, d_tokens, d_parents, d_offsets, d_uniform, sampler, d_path_out, d_n_path_out, d_next_out, d_logprobs_out=None,
                      d_draft_probs=None):
        """rpo_verify_drafts: d_logits and d_draft_probs float32 [rows, vocab] (rows may be strided), d_tokens and d_parents int32 [rows],
        d_offsets int32 [n_seqs + 1], d_uniform float32 [rows], d_path_out int32 [n_seqs, max_path], d_n_path_out and d_next_out
        int32 [n_seqs], d_logprobs_out float32 like d_path_out."""
        dev = d_logits.device
        if self.device is not None and dev != self.device:
            raise ValueError(f"d_logits is on {dev}, the context on {self.device}")
        strides = []
        for t, name in ((d_logits, "d_logits"), (d_draft_probs, "d_draft_probs")):
            if t is None:
                strides.append(0)
                continue
            if t.dim() != 2 or t.dtype is not _dtype("float32") or t.shape != d_logits.shape or t.device != dev or (t.numel() and t.shape[1] > 1 and t.stride(1) != 1):
                raise ValueError(f"{name} must be float32 [rows, vocab] on {dev} with contiguous rows, got {t.dtype} {tuple(t.shape)}")
            strides.append(t.stride(0) if t.shape[0] > 1 else t.shape[1])
        n, vocab = d_logits.shape
        n_seqs = d_offsets.shape[0] - 1
        _expect(d_offsets, "d_offsets", "int32", (n_seqs + 1,), dev)
        _expect(d_tokens, "d_tokens", "int32", (n,), dev)
        _expect(d_parents, "d_parents", "int32", (n,), dev)
        _expect(d_uniform, "d_uniform", "float32", (n,), dev)
        max_path = d_path_out.shape[-1]
        _expect(d_path_out, "d_path_out", "int32", (n_seqs, max_path), dev)
        _expect(d_n_path_out, "d_n_path_out", "int32", (n_seqs,), dev)
        _expect(d_next_out, "d_next_out", "int32", (n_seqs,), dev)
        if d_logprobs_out is not None:
            _expect(d_logprobs_out, "d_logprobs_out", "float32", (n_seqs, max_path), dev)
        _check(self.lib.rpo_verify_drafts(self.handle, n_seqs, n, vocab, d_logits.data_ptr(), strides[0],
                                          None if d_draft_probs is None else d_draft_probs.data_ptr(), strides[1], d_tokens.data_ptr(),
                                          d_parents.data_ptr(), d_offsets.data_ptr(), d_uniform.data_ptr(), C.byref(sampler), max_path,
                                          d_path_out.data_ptr(), d_n_path_out.data_ptr(), d_next_out.data_ptr(),
                                          None if d_logprobs_out is None else d_logprobs_out.data_ptr()), "rpo_verify_drafts")

    def commit_path(self, layers, d_q_offsets, d_path, d_n_path, d_lens_out):
        """rpo_commit_path: layers a PagedLayers, d_q_offsets int32 [n_seqs + 1], d_path int32 [n_seqs, max_path], d_n_path and
        d_lens_out (the caches' d_lens, say) int32 [n_seqs]."""
        self._paged_dtype(layers)
        n = layers.n_seqs
        _expect(d_q_offsets, "d_q_offsets", "int32", (n + 1,), layers.device)
        _expect(d_path, "d_path", "int32", (n, d_path.shape[-1]), layers.device)
        _expect(d_n_path, "d_n_path", "int32", (n,), layers.device)
        _expect(d_lens_out, "d_lens_out", "int32", (n,), layers.device)
        _check(self.lib.rpo_commit_path(self.handle, layers.array, len(layers.layers), d_q_offsets.data_ptr(), d_path.data_ptr(), d_path.shape[-1],
                                        d_n_path.data_ptr(), d_lens_out.data_ptr()), "rpo_commit_path")

    def _page_pool(self, pool, layers):
        self._paged_dtype(layers)
        if pool.device != layers.device or pool.d_block_table.data_ptr() != layers.layers[0].d_block_table.data_ptr():
            raise ValueError("the pool must share its block table with the caches")

    def fork_pages(self, pool, layers, d_src, d_dst, d_fork_lens, d_lens_out=None):
        """rpo_fork_pages: pool a PagePool, layers a PagedLayers, d_src, d_dst, d_fork_lens int32 [forks], d_lens_out int32 [n_seqs]."""
        self._page_pool(pool, layers)
        n = d_src.shape[0]
        for t, name in ((d_src, "d_src"), (d_dst, "d_dst"), (d_fork_lens, "d_fork_lens")):
            _expect(t, name, "int32", (n,), layers.device)
        if d_lens_out is not None:
            _expect(d_lens_out, "d_lens_out", "int32", (layers.n_seqs,), layers.device)
        _check(self.lib.rpo_fork_pages(self.handle, pool.ref, layers.array, len(layers.layers), n, d_src.data_ptr(), d_dst.data_ptr(),
                                       d_fork_lens.data_ptr(), None if d_lens_out is None else d_lens_out.data_ptr()), "rpo_fork_pages")

    def reserve_pages(self, pool, layers, d_lens, d_target_lens):
        """rpo_reserve_pages: d_lens (tokens that stay) and d_target_lens (tokens to hold pages for) int32 [n_seqs]."""
        self._page_pool(pool, layers)
        for t, name in ((d_lens, "d_lens"), (d_target_lens, "d_target_lens")):
            _expect(t, name, "int32", (layers.n_seqs,), layers.device)
        _check(self.lib.rpo_reserve_pages(self.handle, pool.ref, layers.array, len(layers.layers), d_lens.data_ptr(), d_target_lens.data_ptr()),
               "rpo_reserve_pages")

    def attention_mass(self, d_q, kv, d_q_offsets, max_chunk, d_lse, d_mass_out, d_mass_in=None, scale=None, window=0, sinks=0):
        """rpo_attention_mass: d_lse float32 [rows, n_q_heads] of chunk_attention, d_mass_out (and d_mass_in, which may be the same
        tensor) float32 [n_seqs, n_kv_heads, slots]."""
        dt, st = self._paged_dtype(kv), kv.struct
        n, hq = d_q.shape[0], d_q.shape[1]
        q_stride = _head_rows(d_q, "d_q", dt, hq, st.head_dim, kv.device)
        _expect(d_q_offsets, "d_q_offsets", "int32", (st.n_seqs + 1,), kv.device)
        _expect(d_lse, "d_lse", "float32", (n, hq), kv.device)
        slots = d_mass_out.shape[-1]
        _expect(d_mass_out, "d_mass_out", "float32", (st.n_seqs, st.n_kv_heads, slots), kv.device)
        if d_mass_in is not None:
            _expect(d_mass_in, "d_mass_in", "float32", (st.n_seqs, st.n_kv_heads, slots), kv.device)
        cfg = self._chunk_cfg(kv, scale, window, sinks)
        _check(self.lib.rpo_attention_mass(self.handle, kv.ref, n, hq, max_chunk, d_q.data_ptr(), q_stride, d_q_offsets.data_ptr(), C.byref(cfg),
                                           d_lse.data_ptr(), None if d_mass_in is None else d_mass_in.data_ptr(), d_mass_out.data_ptr(), slots),
               "rpo_attention_mass")

    def evict_cache(self, kv, d_mass, d_positions, budget, d_lens_out, d_src_out, d_mass_out, d_positions_out, sinks=0, recent=0):
        """rpo_evict_cache: d_mass float32 and d_positions int32 [n_seqs, n_kv_heads, slots], d_src_out int32 [n_seqs, n_kv_heads,
        budget], d_mass_out / d_positions_out of at least budget slots (or d_mass / d_positions themselves), d_lens_out int32
        [n_seqs] (or the cache's own d_lens; of layers that share one, in the last layer's call only)."""
        self._paged_dtype(kv)
        n, h = kv.struct.n_seqs, kv.struct.n_kv_heads
        slots, out_slots = d_mass.shape[-1], d_mass_out.shape[-1]
        _expect(d_mass, "d_mass", "float32", (n, h, slots), kv.device)
        _expect(d_positions, "d_positions", "int32", (n, h, slots), kv.device)
        _expect(d_lens_out, "d_lens_out", "int32", (n,), kv.device)
        _expect(d_src_out, "d_src_out", "int32", (n, h, budget), kv.device)
        _expect(d_mass_out, "d_mass_out", "float32", (n, h, out_slots), kv.device)
        _expect(d_positions_out, "d_positions_out", "int32", (n, h, out_slots), kv.device)
        _check(self.lib.rpo_evict_cache(self.handle, kv.ref, d_mass.data_ptr(), d_positions.data_ptr(), slots, budget, sinks, recent,
                                        d_lens_out.data_ptr(), d_src_out.data_ptr(), d_mass_out.data_ptr(), d_positions_out.data_ptr(), out_slots),
               "rpo_evict_cache")

    def device_status(self, raise_on_timeout=True):
        """The device status word (cleared by the read).  An expired device-side wait (bit 0) raises
        RpoError(RPO_ERR_DEVICE_TIMEOUT) unless raise_on_timeout is False."""
        v = C.c_int32()
        rc = self.lib.rpo_device_status(self.handle, C.byref(v))
        if rc != 0 and (raise_on_timeout or rc != -5):
            raise RpoError(rc, "rpo_device_status")
        return v.value

    def debug_tap(self, d_buf):
        """Set (tensor) or clear (None) the residual-stream tap; returns the floats written so far."""
        used = C.c_int64()
        _check(self.lib.rpo_debug_tap(self.handle, _ptr(d_buf), 0 if d_buf is None else d_buf.numel(), C.byref(used)),
               "rpo_debug_tap")
        return used.value

    def counters(self):
        a, b = C.c_int64(), C.c_int64()
        _check(self.lib.rpo_counters(self.handle, C.byref(a), C.byref(b)), "rpo_counters")
        return a.value, b.value

    def set_option(self, name, value):
        _check(self.lib.rpo_set_option(self.handle, name.encode(), int(value)), f"rpo_set_option({name})")

    PHASES = ("prefill", "decode", "logprobs")
    CLASSES = ("other", "gemm", "attention", "sampler", "rmsnorm", "rope_kv")

    def profile_read(self):
        """{phase: {class: (total_ms, launches)}} since the last read (needs option profile=1)."""
        n = len(self.PHASES) * len(self.CLASSES)
        ms = (C.c_double * n)(); cnt = (C.c_int64 * n)()
        _check(self.lib.rpo_profile_read(self.handle, ms, cnt, n), "rpo_profile_read")
        return {p: {k: (ms[i * len(self.CLASSES) + j], cnt[i * len(self.CLASSES) + j])
                    for j, k in enumerate(self.CLASSES)} for i, p in enumerate(self.PHASES)}
