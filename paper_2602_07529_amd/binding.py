"""ctypes binding of libdagattn.so: argument marshalling only.

Every step of the path runs in the library's HIP kernels; PyTorch is used for device memory and
for the current stream handle.  There is no CPU fallback: if the library is missing, loading
raises.  Function names match the C ABI declared in include/dagattn.h.
"""
import ctypes as C
import os

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("DAGATTN_LIB") or os.path.join(_PKG, "libdagattn.so")

DAG_F32, DAG_BF16 = 0, 1
DAG_STRICT_CLOSURE = 1
TILE_SKIP, TILE_PARTIAL, TILE_FULL = 0, 1, 2
PAGE = 16
ROPE_HALVES, ROPE_PAIRS = 0, 1


class DagError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("dagattn error %d: %s" % (code, msg))
        self.code = code


class dag_desc_t(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("node_offsets", C.c_void_p), ("node_len", C.c_void_p),
                ("anc_bits", C.c_void_p), ("words_per_node", C.c_int32), ("tile_m", C.c_int32),
                ("tile_n", C.c_int32), ("flags", C.c_uint32)]


class dag_meta_sizes_t(C.Structure):
    _fields_ = [("total_nodes", C.c_int64), ("total_tokens", C.c_int64), ("total_qtiles", C.c_int64),
                ("total_ktiles", C.c_int64), ("total_tiles", C.c_int64), ("csr_capacity", C.c_int64),
                ("workspace_bytes", C.c_int64)]


_META_ARRAYS = [("cu_seqlens", torch.int32), ("node_start", torch.int32), ("tok_node", torch.int32),
                ("pos_ids", torch.int32), ("node_tok_start", torch.int32), ("node_pos_start", torch.int32),
                ("node_vis", torch.int64), ("qtile_start", torch.int32), ("ktile_start", torch.int32),
                ("block_map_off", torch.int64),
                ("block_map", torch.uint8), ("qtile_rowptr", torch.int32), ("qtile_col", torch.int32),
                ("qtile_flag", torch.uint8), ("qtile_nfull", torch.int32), ("qtile_order", torch.int32), ("qtile_desc", torch.int32),
                ("useful_pairs", torch.int64)]


class dag_meta_t(C.Structure):
    _fields_ = ([("n_seqs", C.c_int32), ("words_per_node", C.c_int32), ("tile_m", C.c_int32),
                 ("tile_n", C.c_int32), ("sizes", dag_meta_sizes_t)] +
                [(name, C.c_void_p) for name, _ in _META_ARRAYS])


class dag_decode_desc_t(C.Structure):
    _fields_ = [("n_groups", C.c_int32), ("n_live", C.c_int32), ("page_size", C.c_int32),
                ("max_shared_pages", C.c_int32), ("max_branch_pages", C.c_int32),
                ("max_group_size", C.c_int32),
                ("group_branch_off", C.c_void_p), ("shared_page_off", C.c_void_p),
                ("shared_pages", C.c_void_p), ("shared_len", C.c_void_p),
                ("branch_page_off", C.c_void_p), ("branch_pages", C.c_void_p),
                ("branch_len", C.c_void_p), ("branch_pos", C.c_void_p)]


_SEG_ARRAYS = ("seg_page_off", "seg_pages", "seg_len", "seg_reader_off", "seg_readers", "branch_entry_off",
               "branch_entries")


class dag_decode_seg_desc_t(C.Structure):
    _fields_ = ([("n_live", C.c_int32), ("n_segments", C.c_int32), ("page_size", C.c_int32),
                 ("max_seg_pages", C.c_int32), ("max_readers", C.c_int32), ("total_readers", C.c_int32)] +
                [(name, C.c_void_p) for name in _SEG_ARRAYS] + [("seg_reader_len", C.c_void_p)])


_PAGED_ARRAYS = ("q_off", "ctx_page_off", "ctx_pages", "ctx_page_len", "own_page", "own_len")


class dag_paged_prefill_desc_t(C.Structure):
    _fields_ = ([("n_nodes", C.c_int32), ("page_size", C.c_int32), ("max_new", C.c_int32),
                 ("max_ctx_pages", C.c_int32)] + [(name, C.c_void_p) for name in _PAGED_ARRAYS])


_SCHED_ARRAYS = ("live_node", "live_token", "branch_page_off", "branch_pages", "branch_len", "branch_pos",
                 "seg_node", "seg_page_off", "seg_pages", "seg_len", "seg_reader_off", "seg_readers",
                 "seg_reader_len", "branch_entry_off", "branch_entries")


class dag_sched_step_t(C.Structure):
    _fields_ = ([(name, C.c_int32) for name in ("n_live", "layer", "n_segments", "max_seg_pages", "max_readers",
                                                "total_readers", "n_branch_pages", "n_seg_pages", "pages_in_use")] +
                [(name, C.POINTER(C.c_int32)) for name in _SCHED_ARRAYS])


class dag_kv_q8_t(C.Structure):
    _fields_ = [("k_pool", C.c_void_p), ("v_pool", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("n_pages", C.c_int32), ("hkv", C.c_int32), ("head_dim", C.c_int32)]


class dag_rope_t(C.Structure):
    _fields_ = [("freq", C.c_void_p), ("factor", C.c_double), ("rotary_dim", C.c_int32), ("layout", C.c_int32)]


class dag_kv_rows_t(C.Structure):
    _fields_ = [("n_rows", C.c_int32), ("page_size", C.c_int32), ("max_row_pages", C.c_int32), ("n_pages", C.c_int32),
                ("table", C.c_void_p), ("free_pages", C.c_void_p)]


_lib = None


def lib():
    """Load the shared library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libdagattn.so is not built: run `python -m paper_2602_07529_amd.build` "
                               "(there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
        L.dag_prefill_tile_shape.argtypes = [i32, i32, i32, C.c_int, C.POINTER(i32), C.POINTER(i32)]
        L.dag_meta_sizes.argtypes = [C.POINTER(dag_desc_t), C.POINTER(dag_meta_sizes_t)]
        L.dag_build_meta.argtypes = [C.POINTER(dag_desc_t), C.POINTER(dag_meta_t), vp, C.c_size_t, vp]
        L.dag_rope_qk.argtypes = [vp, i64, vp, vp, i32, i32, i32, f32, C.c_int, vp]
        L.dag_attn_prefill.argtypes = [C.POINTER(dag_meta_t), vp, vp, vp, vp, vp, i32, i32, i32, f32,
                                       C.c_int, vp, C.c_size_t, vp]
        L.dag_attn_prefill_prepared.argtypes = L.dag_attn_prefill.argtypes
        L.dag_prefill_prepare_v.argtypes = [C.POINTER(dag_meta_t), vp, i32, i32, i32, C.c_int, vp, C.c_size_t, vp]
        L.dag_prefill_workspace_bytes.argtypes = [C.POINTER(dag_meta_t), i32, i32, C.c_int]
        L.dag_prefill_workspace_bytes.restype = C.c_size_t
        L.dag_prefill_bwd_workspace_bytes.argtypes = [C.POINTER(dag_meta_t), i32, i32, i32]
        L.dag_prefill_bwd_workspace_bytes.restype = C.c_size_t
        L.dag_attn_prefill_bwd.argtypes = [C.POINTER(dag_meta_t), vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32,
                                           f32, C.c_int, vp, C.c_size_t, vp]
        L.dag_kv_append_rope.argtypes = [C.POINTER(dag_decode_desc_t), vp, vp, vp, vp, i32, i32, f32, vp]
        L.dag_decode_workspace_bytes.argtypes = [C.POINTER(dag_decode_desc_t), i32, i32, i32]
        L.dag_decode_workspace_bytes.restype = C.c_size_t
        L.dag_attn_decode.argtypes = [C.POINTER(dag_decode_desc_t), vp, vp, vp, vp, i32, i32, i32, f32,
                                      vp, C.c_size_t, vp]
        L.dag_attn_decode_static.argtypes = [C.POINTER(dag_decode_desc_t), vp, vp, vp, vp, i32, i32, i32, f32, vp]
        L.dag_decode_segments_workspace_bytes.argtypes = [C.POINTER(dag_decode_seg_desc_t), i32, i32, i32]
        L.dag_decode_segments_workspace_bytes.restype = C.c_size_t
        L.dag_attn_decode_segments.argtypes = [C.POINTER(dag_decode_seg_desc_t), vp, vp, vp, vp, i32, i32, i32, f32,
                                               vp, C.c_size_t, vp]
        L.dag_prefill_paged_workspace_bytes.argtypes = [C.POINTER(dag_paged_prefill_desc_t)]
        L.dag_prefill_paged_workspace_bytes.restype = C.c_size_t
        L.dag_attn_prefill_paged.argtypes = [C.POINTER(dag_paged_prefill_desc_t), vp, vp, vp, i32, vp, vp, i32, i32,
                                             i32, f32, vp, C.c_size_t, vp]
        L.dag_kv_append_rope_q8.argtypes = [C.POINTER(dag_kv_q8_t), vp, vp, i64, vp, vp, f32, C.c_int, vp]
        for name, desc in (("decode_q8", dag_decode_desc_t), ("decode_segments_q8", dag_decode_seg_desc_t)):
            need, call = getattr(L, "dag_%s_workspace_bytes" % name), getattr(L, "dag_attn_" + name)
            need.argtypes, need.restype = [C.POINTER(desc), i32, i32, i32], C.c_size_t
            call.argtypes = [C.POINTER(desc), C.POINTER(dag_kv_q8_t), vp, vp, i32, f32, vp, C.c_size_t, vp]
        L.dag_prefill_paged_q8_workspace_bytes.argtypes = [C.POINTER(dag_paged_prefill_desc_t), i64, i32, i32, i32]
        L.dag_prefill_paged_q8_workspace_bytes.restype = C.c_size_t
        L.dag_attn_prefill_paged_q8.argtypes = [C.POINTER(dag_paged_prefill_desc_t), C.POINTER(dag_kv_q8_t), vp, i64, vp, vp, i32, f32, vp,
                                                C.c_size_t, vp]
        f64 = C.c_double
        L.dag_rope_frequencies.argtypes = [vp, i32, f64, f64, f64, f64, f64]
        L.dag_rope_apply.argtypes = [C.POINTER(dag_rope_t), vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, i32, i32, i32, i32, C.c_int, vp]
        L.dag_kv_append_rotary_q8.argtypes = [C.POINTER(dag_kv_q8_t), vp, vp, i64, vp, i64, vp, i64, C.POINTER(dag_rope_t), C.c_int, vp]
        rows = C.POINTER(dag_kv_rows_t)
        L.dag_kv_pages_workspace_bytes.argtypes = [i32, i32, i32]
        L.dag_kv_pages_workspace_bytes.restype = C.c_size_t
        L.dag_kv_fork.argtypes = [rows, i32] + [vp] * 13 + [C.c_size_t, vp]
        L.dag_kv_release_shared.argtypes = [rows] + [vp] * 8 + [C.c_size_t, vp]
        L.dag_kv_compact.argtypes = [rows, rows] + [vp] * 9 + [C.c_size_t, vp]
        L.dag_kv_copy_pages_q8.argtypes = [C.POINTER(dag_kv_q8_t), vp, vp, i32, vp, vp]
        L.dag_kv_copy_pages.argtypes = [vp, vp, i32, i32, i32, vp, vp, i32, vp, vp]
        L.dag_kv_tables_workspace_bytes.argtypes = [i32]
        L.dag_kv_tables_workspace_bytes.restype = C.c_size_t
        L.dag_kv_release.argtypes = [C.POINTER(dag_kv_rows_t), vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.dag_kv_tables.argtypes = [C.POINTER(dag_kv_rows_t), vp, vp, vp, vp, vp, vp, vp, i64, vp, vp, vp, vp, i64, vp, vp,
                                    C.c_size_t, vp]
        L.dag_copy_calibration.argtypes = [vp, vp, C.c_size_t, vp]
        L.dag_sched_create.argtypes = [i32, vp, vp, vp, vp, i32, i32, C.POINTER(vp)]
        L.dag_sched_destroy.argtypes = [vp]
        L.dag_sched_destroy.restype = None
        L.dag_sched_step.argtypes = [vp, C.POINTER(dag_sched_step_t)]
        L.dag_strerror.argtypes = [C.c_int]
        L.dag_strerror.restype = C.c_char_p
        L.dag_version.restype = C.c_int
        for name in ("dag_prefill_tile_shape", "dag_meta_sizes", "dag_build_meta", "dag_rope_qk",
                     "dag_attn_prefill", "dag_attn_prefill_prepared", "dag_prefill_prepare_v",
                     "dag_kv_append_rope", "dag_attn_decode", "dag_attn_decode_static", "dag_attn_decode_segments",
                     "dag_sched_create", "dag_attn_prefill_paged", "dag_copy_calibration",
                     "dag_attn_prefill_bwd", "dag_kv_append_rope_q8", "dag_attn_decode_q8", "dag_attn_decode_segments_q8",
                     "dag_attn_prefill_paged_q8", "dag_rope_frequencies", "dag_rope_apply", "dag_kv_append_rotary_q8", "dag_kv_fork",
                     "dag_kv_release_shared", "dag_kv_compact", "dag_kv_copy_pages_q8", "dag_kv_copy_pages", "dag_kv_release", "dag_kv_tables",
                     "dag_sched_step"):
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def _check(rc):
    if rc != 0:
        raise DagError(rc, lib().dag_strerror(rc).decode())


def _stream():
    # (the handle without a torch.cuda.Stream object around it: 0.3 instead of 2.9 us a call, of 8 to 11)
    return C.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))


def _ptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else C.c_void_p(0)


def _dtype_code(t):
    if t.dtype == torch.float32:
        return DAG_F32
    if t.dtype == torch.bfloat16:
        return DAG_BF16
    raise TypeError("unsupported dtype %s" % t.dtype)


def dag_strerror(code):
    return lib().dag_strerror(code).decode()


def dag_version():
    return lib().dag_version()


def dag_prefill_tile_shape(hq, hkv, head_dim, dtype_code):
    tm, tn = C.c_int32(0), C.c_int32(0)
    _check(lib().dag_prefill_tile_shape(hq, hkv, head_dim, dtype_code, C.byref(tm), C.byref(tn)))
    return tm.value, tn.value


class DagDesc:
    """Host-side node table (keeps the numpy arrays alive for the ctypes struct)."""

    def __init__(self, node_offsets, node_len, anc_bits, words_per_node, tile_m, tile_n, flags=0):
        self.node_offsets = np.ascontiguousarray(node_offsets, dtype=np.int32)
        self.node_len = np.ascontiguousarray(node_len, dtype=np.int32)
        self.anc_bits = np.ascontiguousarray(anc_bits, dtype=np.uint64)
        self.c = dag_desc_t(len(self.node_offsets) - 1, self.node_offsets.ctypes.data,
                            self.node_len.ctypes.data, self.anc_bits.ctypes.data,
                            words_per_node, tile_m, tile_n, flags)


def dag_meta_sizes(desc):
    out = dag_meta_sizes_t()
    _check(lib().dag_meta_sizes(C.byref(desc.c), C.byref(out)))
    return out


class DagMeta:
    """Device tables written by dag_build_meta (torch tensors + the ctypes struct pointing at them)."""

    def __init__(self, desc, sizes, device):
        n = desc.c.n_seqs
        W = desc.c.words_per_node
        counts = dict(cu_seqlens=n + 1, node_start=n + 1, tok_node=sizes.total_tokens,
                      pos_ids=sizes.total_tokens, node_tok_start=sizes.total_nodes,
                      node_pos_start=sizes.total_nodes, node_vis=sizes.total_nodes * W,
                      qtile_start=n + 1, ktile_start=n + 1, block_map_off=n + 1, block_map=sizes.total_tiles,
                      qtile_rowptr=sizes.total_qtiles + 1, qtile_col=sizes.csr_capacity,
                      qtile_flag=sizes.csr_capacity, qtile_nfull=sizes.total_qtiles, qtile_order=sizes.total_qtiles, qtile_desc=sizes.total_qtiles * 8,
                      useful_pairs=n)
        self.sizes = sizes
        self.t = {name: torch.empty(max(int(counts[name]), 1), dtype=dt, device=device)
                  for name, dt in _META_ARRAYS}
        self.counts = counts
        self.c = dag_meta_t()
        self.c.n_seqs, self.c.words_per_node = n, W
        self.c.tile_m, self.c.tile_n = desc.c.tile_m, desc.c.tile_n
        self.c.sizes = sizes
        for name, _ in _META_ARRAYS:
            setattr(self.c, name, self.t[name].data_ptr())
        self.workspace = torch.empty(max(int(sizes.workspace_bytes), 16), dtype=torch.uint8, device=device)

    def get(self, name):
        """Valid prefix of a table as a torch tensor."""
        return self.t[name][:int(self.counts[name])]


def dag_build_meta(desc, meta):
    _check(lib().dag_build_meta(C.byref(desc.c), C.byref(meta.c), _ptr(meta.workspace),
                                meta.workspace.numel(), _stream()))


def dag_rope_qk(pos_ids, q, k, theta):
    ref = q if q is not None else k
    n_tokens, d = ref.shape[0], ref.shape[-1]
    hq = q.shape[1] if q is not None else 0
    hkv = k.shape[1] if k is not None else 0
    _check(lib().dag_rope_qk(_ptr(pos_ids), n_tokens, _ptr(q), _ptr(k), hq, hkv, d, float(theta),
                             _dtype_code(ref), _stream()))


def dag_prefill_workspace_bytes(meta, hkv, head_dim, dtype_code):
    return int(lib().dag_prefill_workspace_bytes(C.byref(meta.c), hkv, head_dim, dtype_code))


def _prefill_workspace(meta, hkv, d, like, workspace):
    if workspace is not None:
        return workspace
    need = dag_prefill_workspace_bytes(meta, hkv, d, _dtype_code(like))
    ws = getattr(meta, "prefill_ws", None)
    if ws is None or ws.numel() < need:
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=like.device)
        meta.prefill_ws = ws
    return ws


def dag_attn_prefill(meta, q, k, v, out, lse=None, softmax_scale=None, workspace=None, prepared=False):
    """`workspace`: uint8 device tensor of dag_prefill_workspace_bytes(); when omitted one is
    allocated (torch) and kept on `meta` for the following calls.  prepared=True calls
    dag_attn_prefill_prepared (the workspace already holds what dag_prefill_prepare_v wrote)."""
    T, hq, d = q.shape
    hkv = k.shape[1]
    if softmax_scale is None:
        softmax_scale = 1.0 / float(d) ** 0.5
    workspace = _prefill_workspace(meta, hkv, d, q, workspace)
    fn = lib().dag_attn_prefill_prepared if prepared else lib().dag_attn_prefill
    _check(fn(C.byref(meta.c), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), hq, hkv, d, float(softmax_scale),
              _dtype_code(q), _ptr(workspace), workspace.numel(), _stream()))


def dag_prefill_prepare_v(meta, v, hq, workspace=None):
    hkv, d = v.shape[1], v.shape[2]
    workspace = _prefill_workspace(meta, hkv, d, v, workspace)
    _check(lib().dag_prefill_prepare_v(C.byref(meta.c), _ptr(v), hq, hkv, d, _dtype_code(v), _ptr(workspace),
                                       workspace.numel(), _stream()))


_DECODE_ARRAYS = ("group_branch_off", "shared_page_off", "shared_pages", "shared_len", "branch_page_off",
                  "branch_pages", "branch_len", "branch_pos")


def _int32(x, name):
    if x.dtype != torch.int32 or not x.is_contiguous():
        raise TypeError("%s has to be a contiguous int32 tensor" % name)


def _device_arrays(arrays, least=()):
    """int32 tensors on one device, `least` elements long."""
    least, devices = dict(least), set()
    for name, x in arrays.items():
        if x is not None:
            _int32(x, name)
            if x.numel() < least.get(name, 0):
                raise ValueError("%s has %d elements, not %d" % (name, x.numel(), least[name]))
            devices.add(x.device)
    _one_device(devices)
    return arrays


def _one_device(devices):
    if len(devices) > 1:
        raise ValueError("tensors are on %s" % ", ".join(sorted(map(str, devices))))


class DecodeDesc:
    """Device copies of the decode description arrays + the ctypes struct."""

    def __init__(self, desc, device):
        self.t = {}
        for name in ("group_branch_off", "shared_page_off", "shared_pages", "shared_len",
                     "branch_page_off", "branch_pages", "branch_len", "branch_pos"):
            arr = np.ascontiguousarray(desc[name], dtype=np.int32)
            if arr.size == 0:
                arr = np.zeros(1, dtype=np.int32)
            self.t[name] = torch.from_numpy(arr).to(device)
        ng, nl = int(desc["n_groups"]), int(desc["n_live"])
        sp = np.diff(np.asarray(desc["shared_page_off"])) if ng else np.zeros(0)
        bp = np.diff(np.asarray(desc["branch_page_off"])) if nl else np.zeros(0)
        gs = np.diff(np.asarray(desc["group_branch_off"])) if ng else np.zeros(0)
        self.c = dag_decode_desc_t(ng, nl, int(desc["page_size"]),
                                   int(sp.max()) if sp.size else 0, int(bp.max()) if bp.size else 0,
                                   int(gs.max()) if gs.size else 0,
                                   *[self.t[n].data_ptr() for n in
                                     ("group_branch_off", "shared_page_off", "shared_pages", "shared_len",
                                      "branch_page_off", "branch_pages", "branch_len", "branch_pos")])


    @classmethod
    def on_device(cls, n_groups, n_live, max_shared_pages, max_branch_pages, max_group_size, group_branch_off=None,
                  shared_page_off=None, shared_pages=None, shared_len=None, branch_page_off=None, branch_pages=None,
                  branch_len=None, branch_pos=None):
        """A description whose arrays are on the device already (int32 tensors, kept alive here), with the host bounds."""
        self = cls.__new__(cls)
        arrays = (group_branch_off, shared_page_off, shared_pages, shared_len, branch_page_off, branch_pages, branch_len,
                  branch_pos)
        self.t = _device_arrays(dict(zip(_DECODE_ARRAYS, arrays)), dict(
            group_branch_off=n_groups + 1, shared_page_off=n_groups + 1, shared_len=n_groups, branch_page_off=n_live + 1,
            branch_len=n_live, branch_pos=n_live) if n_groups else dict(branch_page_off=n_live + 1, branch_len=n_live, branch_pos=n_live))
        self.c = dag_decode_desc_t(n_groups, n_live, PAGE, max_shared_pages, max_branch_pages, max_group_size,
                                   *[0 if x is None else x.data_ptr() for x in arrays])
        return self


def dag_kv_append_rope(ddesc, k_new, v_new, k_pool, v_pool, theta):
    hkv, d = k_new.shape[1], k_new.shape[2]
    _check(lib().dag_kv_append_rope(C.byref(ddesc.c), _ptr(k_new), _ptr(v_new), _ptr(k_pool), _ptr(v_pool),
                                    hkv, d, float(theta), _stream()))


def dag_decode_workspace_bytes(ddesc, hq, hkv, head_dim):
    return int(lib().dag_decode_workspace_bytes(C.byref(ddesc.c), hq, hkv, head_dim))


def dag_attn_decode(ddesc, q, k_pool, v_pool, out, workspace, softmax_scale=None):
    n_live, hq, d = q.shape
    hkv = k_pool.shape[1]
    if softmax_scale is None:
        softmax_scale = 1.0 / float(d) ** 0.5
    _check(lib().dag_attn_decode(C.byref(ddesc.c), _ptr(q), _ptr(k_pool), _ptr(v_pool), _ptr(out), hq, hkv, d,
                                 float(softmax_scale), _ptr(workspace), workspace.numel(), _stream()))


DECODE_STATIC_SCRATCH_BYTES = 32 << 20


def dag_attn_decode_static(ddesc, q, k_pool, v_pool, out, softmax_scale=None):
    """dag_attn_decode without a workspace: the partial results live in the library's own device
    array (DAG_ERR_WORKSPACE when the description needs more than DECODE_STATIC_SCRATCH_BYTES)."""
    n_live, hq, d = q.shape
    hkv = k_pool.shape[1]
    if softmax_scale is None:
        softmax_scale = 1.0 / float(d) ** 0.5
    _check(lib().dag_attn_decode_static(C.byref(ddesc.c), _ptr(q), _ptr(k_pool), _ptr(v_pool), _ptr(out), hq, hkv, d,
                                        float(softmax_scale), _stream()))


class SegDecodeDesc:
    """Device copies of the segment-form decode description arrays + the ctypes struct."""

    def __init__(self, desc, device):
        self.t = {}
        for name in _SEG_ARRAYS:
            arr = np.ascontiguousarray(desc[name], dtype=np.int32)
            if arr.size == 0:
                arr = np.zeros(1, dtype=np.int32)
            self.t[name] = torch.from_numpy(arr).to(device)
        ns, nl = int(desc["n_segments"]), int(desc["n_live"])
        sp = np.diff(np.asarray(desc["seg_page_off"])) if ns else np.zeros(0)
        rd = np.diff(np.asarray(desc["seg_reader_off"])) if ns else np.zeros(0)
        self.c = dag_decode_seg_desc_t(nl, ns, int(desc["page_size"]),
                                       int(sp.max()) if sp.size else 0, int(rd.max()) if rd.size else 0,
                                       int(rd.sum()) if rd.size else 0,
                                       *[self.t[n].data_ptr() for n in _SEG_ARRAYS], None)
        if desc.get("seg_reader_len") is not None:
            arr = np.ascontiguousarray(desc["seg_reader_len"], dtype=np.int32)
            self.t["seg_reader_len"] = torch.from_numpy(arr if arr.size else np.zeros(1, np.int32)).to(device)
            self.c.seg_reader_len = self.t["seg_reader_len"].data_ptr()


    @classmethod
    def on_device(cls, n_live, n_segments, max_seg_pages, max_readers, total_readers, seg_page_off, seg_pages, seg_len,
                  seg_reader_off, seg_readers, branch_entry_off, branch_entries, seg_reader_len=None):
        """A description whose arrays are on the device already (int32 tensors, kept alive here), with the host bounds."""
        self = cls.__new__(cls)
        arrays = (seg_page_off, seg_pages, seg_len, seg_reader_off, seg_readers, branch_entry_off, branch_entries,
                  seg_reader_len)
        self.t = _device_arrays(dict(zip(_SEG_ARRAYS + ("seg_reader_len",), arrays)), dict(
            seg_page_off=n_segments + 1, seg_len=n_segments, seg_reader_off=n_segments + 1, branch_entry_off=n_live + 1,
            seg_reader_len=total_readers))
        self.c = dag_decode_seg_desc_t(n_live, n_segments, PAGE, max_seg_pages, max_readers, total_readers,
                                       *[0 if x is None else x.data_ptr() for x in arrays])
        return self


def dag_decode_segments_workspace_bytes(sdesc, hq, hkv, head_dim):
    return int(lib().dag_decode_segments_workspace_bytes(C.byref(sdesc.c), hq, hkv, head_dim))


def dag_attn_decode_segments(sdesc, q, k_pool, v_pool, out, workspace, softmax_scale=None):
    n_live, hq, d = q.shape
    hkv = k_pool.shape[1]
    if softmax_scale is None:
        softmax_scale = 1.0 / float(d) ** 0.5
    _check(lib().dag_attn_decode_segments(C.byref(sdesc.c), _ptr(q), _ptr(k_pool), _ptr(v_pool), _ptr(out), hq, hkv,
                                          d, float(softmax_scale), _ptr(workspace), workspace.numel(), _stream()))


def dag_copy_calibration(dst, src):
    """Plain copy by the library's own kernel (the reference point of the HBM counters)."""
    _check(lib().dag_copy_calibration(_ptr(dst), _ptr(src), src.numel() * src.element_size(), _stream()))


class PagedPrefillDesc:
    """Device copies of the paged-prefill description arrays + the ctypes struct.  `desc`: dict with the six
    arrays of dag_paged_prefill_desc_t (host, int32) and page_size."""

    def __init__(self, desc, device):
        self.t = {}
        for name in _PAGED_ARRAYS:
            arr = np.ascontiguousarray(desc[name], dtype=np.int32)
            self.t[name] = torch.from_numpy(arr if arr.size else np.zeros(1, np.int32)).to(device)
        q_off = np.asarray(desc["q_off"])
        p_off = np.asarray(desc["ctx_page_off"])
        n_nodes = len(q_off) - 1
        self.n_rows = int(q_off[-1])
        self.c = dag_paged_prefill_desc_t(n_nodes, int(desc["page_size"]),
                                          int(np.diff(q_off).max()) if n_nodes else 0,
                                          int(np.diff(p_off).max()) if n_nodes else 0,
                                          *[self.t[n].data_ptr() for n in _PAGED_ARRAYS])

    @classmethod
    def on_device(cls, n_nodes, max_new, max_ctx_pages, q_off, ctx_page_off, ctx_pages, ctx_page_len, own_page, own_len):
        """A description whose arrays are on the device already (int32 tensors, kept alive here), with the host bounds."""
        self = cls.__new__(cls)
        self.t = _device_arrays(dict(zip(_PAGED_ARRAYS, (q_off, ctx_page_off, ctx_pages, ctx_page_len, own_page, own_len))), dict(
            q_off=n_nodes + 1, ctx_page_off=n_nodes + 1, own_page=n_nodes, own_len=n_nodes))
        if ctx_pages.numel() != ctx_page_len.numel():
            raise ValueError("ctx_pages and ctx_page_len are of one length")
        self.n_rows = None  # (known on the device only)
        self.c = dag_paged_prefill_desc_t(n_nodes, PAGE, max_new, max_ctx_pages, *[x.data_ptr() for x in self.t.values()])
        return self


def dag_prefill_paged_workspace_bytes(pdesc):
    return int(lib().dag_prefill_paged_workspace_bytes(C.byref(pdesc.c)))


def dag_attn_prefill_paged(pdesc, q, k_pool, v_pool, out, workspace, lse=None, softmax_scale=None):
    _, hq, d = q.shape
    hkv = k_pool.shape[1]
    if softmax_scale is None:
        softmax_scale = 1.0 / float(d) ** 0.5
    _check(lib().dag_attn_prefill_paged(C.byref(pdesc.c), _ptr(q), _ptr(k_pool), _ptr(v_pool), k_pool.shape[0],
                                        _ptr(out), _ptr(lse) if lse is not None else None, hq, hkv, d,
                                        float(softmax_scale), _ptr(workspace), workspace.numel(), _stream()))


class KvCacheQ8:
    """The tensors of an 8-bit cache (kept alive here) + the ctypes struct.  k_pool [P][hkv][d/16][16][16] and v_pool
    [P][hkv][d][16] float8_e4m3fn, k_scale / v_scale [P][hkv] float32."""

    def __init__(self, k_pool, v_pool, k_scale, v_scale):
        p, hkv, d = v_pool.shape[:3]
        if tuple(k_pool.shape) != (p, hkv, d // 16, PAGE, 16) or tuple(v_pool.shape) != (p, hkv, d, PAGE):
            raise ValueError("pools are [pages][heads][dim / 16][16][16] and [pages][heads][dim][16]")
        if tuple(k_scale.shape) != (p, hkv) or tuple(v_scale.shape) != (p, hkv):
            raise ValueError("scales are [pages][heads]")
        for x, dt in ((k_pool, torch.float8_e4m3fn), (v_pool, torch.float8_e4m3fn), (k_scale, torch.float32),
                      (v_scale, torch.float32)):
            if x.dtype != dt or not x.is_contiguous():
                raise TypeError("pools are contiguous float8_e4m3fn, scales contiguous float32")
        _one_device({k_pool.device, v_pool.device, k_scale.device, v_scale.device})
        self.k_pool, self.v_pool, self.k_scale, self.v_scale = k_pool, v_pool, k_scale, v_scale
        self.hkv, self.head_dim = hkv, d
        self.c = dag_kv_q8_t(k_pool.data_ptr(), v_pool.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), p, hkv, d)
        self.ref = C.byref(self.c)

    @classmethod
    def empty(cls, n_pages, hkv, head_dim, device):
        """A cache without tokens (zeros, scales one)."""
        pool = lambda *shape: torch.zeros((n_pages, hkv) + shape, dtype=torch.uint8, device=device).view(  # noqa: E731
            torch.float8_e4m3fn)
        one = lambda: torch.ones((n_pages, hkv), dtype=torch.float32, device=device)  # noqa: E731
        return cls(pool(head_dim // 16, PAGE, 16), pool(head_dim, PAGE), one(), one())


def _here(*tensors):
    """The current stream's handle; every tensor has to be on its device."""
    here = torch.cuda.current_device()
    for x in tensors:
        if x.get_device() != here and x.numel():
            raise ValueError("tensors have to be on the current device, cuda:%d: got %s" % (here, x.device))
    return torch._C._cuda_getCurrentRawStream(here)


def dag_kv_append_rope_q8(cache, slots, pos, k_new, v_new, theta):
    n = slots.numel()
    shape = (n, cache.hkv, cache.head_dim)
    if k_new.shape != shape or v_new.shape != shape or pos.numel() != n or k_new.dtype != v_new.dtype:
        raise ValueError("k_new and v_new are [tokens][%d][%d] of one type, slots and pos as long" % shape[1:])
    if not k_new.is_contiguous() or not v_new.is_contiguous():
        raise ValueError("k_new and v_new have to be contiguous")
    _int32(slots, "slots")
    _int32(pos, "pos")
    _check(lib().dag_kv_append_rope_q8(cache.ref, slots.data_ptr(), pos.data_ptr(), n, k_new.data_ptr(), v_new.data_ptr(),
                                       theta, _dtype_code(k_new), _here(slots, pos, k_new, v_new, cache.k_pool)))


class Rope:
    """Rotary positions: the table of frequencies on the device (dag_rope_frequencies, or `freq`, a sequence of rotary_dim / 2 of them)
    and the ctypes struct."""

    def __init__(self, rotary_dim, theta, device, layout=ROPE_HALVES, stretch=1.0, original=0.0, low=1.0, high=32.0, factor=1.0, freq=None):
        if freq is None:
            table = np.empty(max(rotary_dim // 2, 1), dtype=np.float64)
            _check(lib().dag_rope_frequencies(table.ctypes.data, rotary_dim, theta, stretch, original, low, high))
        else:
            table = np.ascontiguousarray(freq, dtype=np.float64)
            if table.shape != (rotary_dim // 2,):
                raise ValueError("%d frequencies, not %d" % (table.size, rotary_dim // 2))
        self.freq = torch.from_numpy(table).to(device)
        self.rotary_dim, self.layout, self.factor = rotary_dim, layout, factor
        self.c = dag_rope_t(self.freq.data_ptr(), factor, rotary_dim, layout)
        self.ref = C.byref(self.c)


def _token_stride(x, name):
    """Elements from a token of x [tokens][heads][dim] to the next; its heads lie next to each other."""
    if x.is_contiguous() and x.dim() == 3:
        return x.shape[1] * x.shape[2]
    if x.dim() != 3 or x.stride(2) != 1 or (x.shape[1] > 1 and x.stride(1) != x.shape[2]):
        raise ValueError("%s is [tokens][heads][dim] with the heads of a token next to each other" % name)
    return x.stride(0) if x.shape[0] > 1 else max(x.stride(0), x.shape[1] * x.shape[2])


def dag_rope_apply(rope, pos, q, k, q_out=None, k_out=None, transposed=False):
    """q and k (either may be None) into q_out and k_out, in place without them."""
    ref = q if q is not None else k
    if ref is None:
        return
    n, d, dtype, args, there = pos.numel(), ref.shape[-1], ref.dtype, [], [pos, rope.freq]
    _int32(pos, "pos")
    for name, x, y in (("q", q, q_out), ("k", k, k_out)):
        if x is None:
            if y is not None:
                raise ValueError("%s_out without %s" % (name, name))
            args += (None, 0, None, 0)
            continue
        shape, stride = x.shape, _token_stride(x, name)
        if shape[0] != n or shape[2] != d:
            raise ValueError("%s is [%d][heads][%d]" % (name, n, d))
        if y is None:
            args += (x.data_ptr(), stride, x.data_ptr(), stride)
        else:
            if y.shape != shape:
                raise ValueError("%s_out has the shape of %s" % (name, name))
            args += (x.data_ptr(), stride, y.data_ptr(), _token_stride(y, name + "_out"))
            there.append(y)
        there.append(x)
    for x in there[2:]:
        if x.dtype is not dtype:
            raise TypeError("tensors of one type")
    _check(lib().dag_rope_apply(rope.ref, pos.data_ptr(), n, *args, 0 if q is None else q.shape[1], 0 if k is None else k.shape[1], d, int(transposed),
                                _dtype_code(ref), _here(*there)))


def dag_kv_append_rotary_q8(cache, slots, pos, k_new, v_new, rope):
    n = slots.numel()
    shape = (n, cache.hkv, cache.head_dim)
    if k_new.shape != shape or v_new.shape != shape or pos.numel() != n or k_new.dtype != v_new.dtype:
        raise ValueError("k_new and v_new are [tokens][%d][%d] of one type, slots and pos as long" % shape[1:])
    _int32(slots, "slots")
    _int32(pos, "pos")
    _check(lib().dag_kv_append_rotary_q8(
        cache.ref, slots.data_ptr(), pos.data_ptr(), n, k_new.data_ptr(), _token_stride(k_new, "k_new"), v_new.data_ptr(),
        _token_stride(v_new, "v_new"), rope.ref, _dtype_code(k_new), _here(slots, pos, k_new, v_new, cache.k_pool, rope.freq)))


def dag_decode_q8_workspace_bytes(ddesc, cache, hq):
    return lib().dag_decode_q8_workspace_bytes(C.byref(ddesc.c), hq, cache.hkv, cache.head_dim)


def dag_decode_segments_q8_workspace_bytes(sdesc, cache, hq):
    return lib().dag_decode_segments_q8_workspace_bytes(C.byref(sdesc.c), hq, cache.hkv, cache.head_dim)


def _decode_q8(call, desc, q, cache, out, workspace, softmax_scale):
    n, hq, d = q.shape
    if n != desc.c.n_live or d != cache.head_dim or out.shape != q.shape:
        raise ValueError("q and out are [n_live][heads][head_dim]")
    if q.dtype != torch.bfloat16 or out.dtype != torch.bfloat16 or not q.is_contiguous() or not out.is_contiguous():
        raise TypeError("q and out are contiguous bfloat16")
    array = next((x for x in desc.t.values() if x is not None), q)  # (its arrays are on one device)
    _check(call(desc.c, cache.ref, q.data_ptr(), out.data_ptr(), hq, d ** -0.5 if softmax_scale is None else softmax_scale,
                workspace.data_ptr(), workspace.numel(), _here(q, out, cache.k_pool, workspace, array)))


def dag_attn_decode_q8(ddesc, q, cache, out, workspace, softmax_scale=None):
    _decode_q8(lib().dag_attn_decode_q8, ddesc, q, cache, out, workspace, softmax_scale)


def dag_attn_decode_segments_q8(sdesc, q, cache, out, workspace, softmax_scale=None):
    _decode_q8(lib().dag_attn_decode_segments_q8, sdesc, q, cache, out, workspace, softmax_scale)


def dag_prefill_paged_q8_workspace_bytes(pdesc, cache, n_rows, hq):
    return lib().dag_prefill_paged_q8_workspace_bytes(C.byref(pdesc.c), n_rows, hq, cache.hkv, cache.head_dim)


def dag_attn_prefill_paged_q8(pdesc, q, cache, out, workspace, lse=None, softmax_scale=None):
    n, hq, d = q.shape
    if d != cache.head_dim or out.shape != q.shape:
        raise ValueError("q and out are [rows][heads][head_dim]")
    if pdesc.n_rows is not None and pdesc.n_rows > n:
        raise ValueError("q has %d rows, not the %d of the description" % (n, pdesc.n_rows))
    if q.dtype != torch.bfloat16 or out.dtype != torch.bfloat16 or not q.is_contiguous() or not out.is_contiguous():
        raise TypeError("q and out are contiguous bfloat16")
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous()):
        raise TypeError("lse is contiguous float32 [rows][heads]")
    more = (workspace,) if lse is None else (workspace, lse)
    _check(lib().dag_attn_prefill_paged_q8(
        C.byref(pdesc.c), cache.ref, q.data_ptr(), n, out.data_ptr(), None if lse is None else lse.data_ptr(), hq,
        d ** -0.5 if softmax_scale is None else softmax_scale, workspace.data_ptr(), workspace.numel(),
        _here(q, out, cache.k_pool, pdesc.t["q_off"], *more)))


class KvRows:
    """The page table of rows that grow: table [rows][width] and the stack of free pages [pages], int32 (kept alive here), the
    ctypes struct and the calls' workspace (calls that overlap need rows objects of their own)."""

    def __init__(self, table, free_pages):
        self.table, self.free_pages = table, free_pages
        _device_arrays({"table": table, "free_pages": free_pages})
        n_rows, width = table.shape
        self.c = dag_kv_rows_t(n_rows, PAGE, width, free_pages.numel(), table.data_ptr(), free_pages.data_ptr())
        self.workspace = torch.zeros(int(lib().dag_kv_tables_workspace_bytes(n_rows)), dtype=torch.uint8, device=table.device)
        self.shared_workspaces, self.shared_forks = [], 0  # of the calls on shared pages, the last one in use; forks that it has room for

    def for_shared(self, n_forks=0):
        """The workspace of dag_kv_fork, dag_kv_release_shared and dag_kv_compact, made at the first of them (outside a capture).  A call with
        more forks than it has room for gets a larger one, and the old one is kept: graphs that were captured before go on writing to it."""
        if not self.shared_workspaces or n_forks > self.shared_forks:
            self.shared_forks = max(n_forks, self.c.n_rows, 2 * self.shared_forks)
            need = int(lib().dag_kv_pages_workspace_bytes(self.c.n_rows, self.c.n_pages, self.shared_forks))
            self.shared_workspaces.append(torch.empty(need, dtype=torch.uint8, device=self.table.device))
        return self.shared_workspaces[-1]


def _at(x):
    return 0 if x is None else x.data_ptr()


def _ints(n, **arrays):
    """int32 tensors of n elements each."""
    for name, x in arrays.items():
        if x.numel() != n:
            raise ValueError("%s has %d elements, not %d" % (name, x.numel(), n))
        _int32(x, name)


def dag_kv_release(rows, ended, row_len, row_len_out, free_count, free_count_out):
    _ints(rows.c.n_rows, ended=ended, row_len=row_len, row_len_out=row_len_out)
    _ints(1, free_count=free_count, free_count_out=free_count_out)
    _check(lib().dag_kv_release(rows.c, ended.data_ptr(), row_len.data_ptr(), row_len_out.data_ptr(), free_count.data_ptr(),
                                free_count_out.data_ptr(), rows.workspace.data_ptr(), rows.workspace.numel(),
                                _here(rows.table, ended, row_len, row_len_out, free_count, free_count_out)))


def dag_kv_tables(rows, new_len, row_len, row_len_out, free_count, free_count_out, new_off, slots, pos0=None, pos=None,
                  page_off=None, pages=None, refused=None):
    """`pos` is as long as `slots`; entries past the ends of `slots` and `pages` are dropped."""
    n_rows, n_slots, n_pages = rows.c.n_rows, slots.numel(), 0
    _ints(n_rows, new_len=new_len, row_len=row_len, row_len_out=row_len_out)
    _ints(1, free_count=free_count, free_count_out=free_count_out)
    _ints(n_rows + 1, new_off=new_off)
    _int32(slots, "slots")
    optional = [x for x in (pos0, pos, page_off, pages, refused) if x is not None]
    if pos0 is not None:
        _ints(n_rows, pos0=pos0)
    if pos is not None:
        _ints(n_slots, pos=pos)
    if page_off is not None:
        _ints(n_rows + 1, page_off=page_off)
    if pages is not None:
        n_pages = pages.numel()
        _int32(pages, "pages")
    if refused is not None:
        _ints(1, refused=refused)
    _check(lib().dag_kv_tables(rows.c, new_len.data_ptr(), row_len.data_ptr(), row_len_out.data_ptr(), free_count.data_ptr(),
                               free_count_out.data_ptr(), new_off.data_ptr(), slots.data_ptr(), n_slots, _at(pos0), _at(pos),
                               _at(page_off), _at(pages), n_pages, _at(refused), rows.workspace.data_ptr(),
                               rows.workspace.numel(),
                               _here(rows.table, new_len, row_len, row_len_out, free_count, free_count_out, new_off, slots,
                                     *optional)))


def dag_kv_fork(rows, parent, child, row_len, row_len_out, extra, extra_out, free_count, free_count_out, copy_src, copy_dst, fork_len=None,
                refused=None):
    n, r, p, width = parent.numel(), rows.c.n_rows, rows.c.n_pages, rows.table.numel()
    at, stream = _ints_here(_FORK, (parent, child, fork_len, row_len, row_len_out, extra, extra_out, free_count, free_count_out, copy_src, copy_dst,
                                    refused, rows.table), (n, n, n, r, r, p, p, 1, 1, n, n, 1, width))
    ws = rows.for_shared(n)
    _check(lib().dag_kv_fork(rows.c, n, *at[:-1], ws.data_ptr(), ws.numel(), stream))


def dag_kv_release_shared(rows, ended, row_len, row_len_out, extra, extra_out, free_count, free_count_out):
    r, p = rows.c.n_rows, rows.c.n_pages
    at, stream = _ints_here(_RELEASE_SHARED, (ended, row_len, row_len_out, extra, extra_out, free_count, free_count_out, rows.table),
                            (r, r, r, p, p, 1, 1, rows.table.numel()))
    ws = rows.for_shared()
    _check(lib().dag_kv_release_shared(rows.c, *at[:-1], ws.data_ptr(), ws.numel(), stream))


def dag_kv_compact(rows, rows_out, row_len, extra, extra_out, free_count, page_map, copy_src, copy_dst, n_copies):
    """rows_out may be rows."""
    r, p = rows.c.n_rows, rows.c.n_pages
    at, stream = _ints_here(_COMPACT, (row_len, extra, extra_out, free_count, page_map, copy_src, copy_dst, n_copies, rows.table, rows_out.table),
                            (r, p, p, 1, p, p // 2, p // 2, 1, rows.table.numel(), rows_out.table.numel()))
    ws = rows.for_shared()
    _check(lib().dag_kv_compact(rows.c, rows_out.c, *at[:-2], ws.data_ptr(), ws.numel(), stream))


def _ints_here(names, tensors, counts):
    """_ints and _here for many tensors in one pass (0.4 instead of 1.1 us each); None is left out.  Their pointers and the stream."""
    at, devices = [], set()
    for name, x, n in zip(names, tensors, counts):
        if x is None:
            at.append(0)
            continue
        if x.dtype is not torch.int32 or x.numel() != n or not x.is_contiguous():
            _ints(n, **{name: x})
        if n:
            devices.add(x.get_device())
        at.append(x.data_ptr())
    here = torch.cuda.current_device()
    if devices and devices != {here}:
        _here(*(x for x in tensors if x is not None))
    return at, torch._C._cuda_getCurrentRawStream(here)


_FORK = ("parent", "child", "fork_len", "row_len", "row_len_out", "extra", "extra_out", "free_count", "free_count_out", "copy_src", "copy_dst", "refused",
         "table")
_RELEASE_SHARED = ("ended", "row_len", "row_len_out", "extra", "extra_out", "free_count", "free_count_out", "table")
_COMPACT = ("row_len", "extra", "extra_out", "free_count", "page_map", "copy_src", "copy_dst", "n_copies", "table", "table of rows_out")


def _copies(src, dst, count, pool):
    n = src.numel()
    at, stream = _ints_here(("src", "dst", "count"), (src, dst, count), (n, n, 1))
    if pool.get_device() != torch.cuda.current_device():
        _here(pool)
    return at[0], at[1], n, at[2], stream


def dag_kv_copy_pages_q8(cache, src, dst, count=None):
    """Pages src[i] to dst[i] for all entries, or the first count[0] of them."""
    _check(lib().dag_kv_copy_pages_q8(cache.ref, *_copies(src, dst, count, cache.k_pool)))


def dag_kv_copy_pages(k_pool, v_pool, src, dst, count=None):
    """The same for bf16 pools, [pages][heads][d / 8][16][8] and [pages][heads][d][16]."""
    n_pages, hkv, d = v_pool.shape[:3]
    if tuple(v_pool.shape[3:]) != (PAGE,) or tuple(k_pool.shape) != (n_pages, hkv, d // 8, PAGE, 8):
        raise ValueError("pools are [pages][heads][dim / 8][16][8] and [pages][heads][dim][16]")
    if any(x.dtype != torch.bfloat16 or not x.is_contiguous() for x in (k_pool, v_pool)):
        raise TypeError("pools are contiguous bfloat16")
    _one_device({k_pool.device, v_pool.device})
    _check(lib().dag_kv_copy_pages(k_pool.data_ptr(), v_pool.data_ptr(), n_pages, hkv, d, *_copies(src, dst, count, k_pool)))


class Scheduler:
    """dag_sched_*: the host-side scheduler of the execution phase.  step() returns a dict of
    numpy copies of the step's arrays (None when the net is finished)."""

    def __init__(self, parents, node_len, n_pages, chunk=None, page_size=16):
        n = len(parents)
        off = np.zeros(n + 1, dtype=np.int32)
        off[1:] = np.cumsum([len(p) for p in parents])
        flat = np.asarray([x for p in parents for x in p] or [0], dtype=np.int32)
        ln = np.ascontiguousarray(node_len, dtype=np.int32)
        ch = None if chunk is None else np.ascontiguousarray(chunk, dtype=np.int32)
        self.h = C.c_void_p()
        _check(lib().dag_sched_create(n, off.ctypes.data, flat.ctypes.data, ln.ctypes.data if n else None,
                                      None if ch is None else ch.ctypes.data, int(n_pages), int(page_size),
                                      C.byref(self.h)))

    def step(self):
        st = dag_sched_step_t()
        _check(lib().dag_sched_step(self.h, C.byref(st)))
        if st.n_live == 0:
            return None
        sizes = dict(live_node=st.n_live, live_token=st.n_live, branch_page_off=st.n_live + 1,
                     branch_pages=st.n_branch_pages, branch_len=st.n_live, branch_pos=st.n_live,
                     seg_node=st.n_segments, seg_page_off=st.n_segments + 1, seg_pages=st.n_seg_pages,
                     seg_len=st.n_segments, seg_reader_off=st.n_segments + 1, seg_readers=st.total_readers,
                     seg_reader_len=st.total_readers, branch_entry_off=st.n_live + 1,
                     branch_entries=st.total_readers)
        out = {k: np.ctypeslib.as_array(getattr(st, k), shape=(n,)).copy() if n else np.zeros(0, np.int32)
               for k, n in sizes.items()}
        out.update(n_live=st.n_live, layer=st.layer, n_segments=st.n_segments, page_size=16,
                   pages_in_use=st.pages_in_use)
        return out

    def close(self):
        if self.h:
            lib().dag_sched_destroy(self.h)
            self.h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def dag_prefill_bwd_workspace_bytes(meta, hq, hkv, head_dim):
    return int(lib().dag_prefill_bwd_workspace_bytes(C.byref(meta.c), hq, hkv, head_dim))


def dag_attn_prefill_bwd(meta, q, k, v, out, dout, lse, dq, dk, dv, softmax_scale=None, workspace=None):
    T, hq, d = q.shape
    hkv = k.shape[1]
    if softmax_scale is None:
        softmax_scale = 1.0 / float(d) ** 0.5
    if workspace is None:
        workspace = torch.empty(int(lib().dag_prefill_bwd_workspace_bytes(C.byref(meta.c), hq, hkv, d)),
                                dtype=torch.uint8, device=q.device)
    _check(lib().dag_attn_prefill_bwd(C.byref(meta.c), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(dout), _ptr(lse),
                                      _ptr(dq), _ptr(dk), _ptr(dv), hq, hkv, d, float(softmax_scale),
                                      _dtype_code(q), _ptr(workspace), workspace.numel(), _stream()))
