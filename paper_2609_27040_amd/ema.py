"""Thin ctypes binding of libema_slice.so -- argument marshalling only.

Each function has the C entry point's name without the ``ema_`` prefix and
passes its arguments straight through: torch tensors as their device address
(``data_ptr()``), numpy arrays as host pointers, streams as their hipStream_t.
Before a pointer goes to an entry point that launches kernels, the binding
checks that it is a contiguous GPU tensor of the expected type and at least
the size the call implies (a kernel would dereference a host address or read
past a short tensor); host-only slices take numpy arrays. Every step of the
hot path runs in the library's HIP kernels; there is no fallback. If the
library has not been built this module raises on import.
"""
import ctypes
import os

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib", "libema_slice.so")

OK, ERR_INVAL, ERR_NOMEM, ERR_OWNER, ERR_HIP = 0, -1, -2, -3, -4
F16, BF16, F32 = 0, 1, 2
FULL_WEIGHTS = 0x100
LAYOUT_ATTN, LAYOUT_NHD = 0, 1
ENGINE_KERNEL, ENGINE_DMA = 0, 1
SLAB_LAYER_MAJOR, SLAB_SLAB_MAJOR, SLAB_GROUP_MAJOR = 0, 1, 2
BORROWED = -4
POOL_LOCAL, POOL_SLICE = 0, 1
FREE, STAGING, LENDER = -1, -2, -3
CREATE_HOST_ONLY, CREATE_CHECKED, CREATE_ATTN_GRID = 1, 2, 4
DTYPES = {"f16": F16, "bf16": BF16}


class EmaError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"ema error {code}: {msg}")
        self.code = code


class KVShape(ctypes.Structure):
    _fields_ = [("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("block_size", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("slice_layout", ctypes.c_int32)]


class SliceInfo(ctypes.Structure):
    _fields_ = [("block_bytes", ctypes.c_int64), ("n_local", ctypes.c_int32),
                ("n_slice", ctypes.c_int32), ("lim", ctypes.c_int32),
                ("free_local", ctypes.c_int32), ("free_slice", ctypes.c_int32),
                ("device", ctypes.c_int32), ("local_base", ctypes.c_void_p),
                ("slice_base", ctypes.c_void_p)]


class ReclaimResult(ctypes.Structure):
    _fields_ = [("reclaimed", ctypes.c_int32), ("moved", ctypes.c_int32),
                ("written_back", ctypes.c_int32), ("n_victims", ctypes.c_int32),
                ("lim", ctypes.c_int32)]


class SlabCfg(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int32), ("slab_blocks", ctypes.c_int32),
                ("group", ctypes.c_int32), ("layout", ctypes.c_int32)]


class SlabInfo(ctypes.Structure):
    _fields_ = [("n_slabs", ctypes.c_int32), ("layers", ctypes.c_int32),
                ("slab_blocks", ctypes.c_int32), ("group", ctypes.c_int32),
                ("layout", ctypes.c_int32), ("borrowed", ctypes.c_int32)]


class SlabReclaimResult(ctypes.Structure):
    _fields_ = [("reclaimed", ctypes.c_int32), ("n_victims", ctypes.c_int32),
                ("released", ctypes.c_int32)]


class KVTablesArgs(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in (
        "block_ids", "seq_lens", "new_lens", "staging_ids", "canon_table", "block_table",
        "query_start", "slot_map", "prefetch_src", "prefetch_dst", "prefetch_n", "writeback_src",
        "writeback_dst", "writeback_n")]
        + [(n, ctypes.c_int32) for n in ("layers", "batch", "max_blocks", "n_ids", "n_slots",
                                         "staging_slots", "stage_n", "writeback_cap")])


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                          "(python -m paper_2609_27040_amd.build)")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, I64, SZ, U32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_uint32
    F32C, PSZ = ctypes.c_float, ctypes.POINTER(ctypes.c_size_t)
    sig = {
        "ema_slice_create": [ctypes.POINTER(KVShape), SZ, SZ, U32, ctypes.POINTER(P)],
        "ema_slice_destroy": [P],
        "ema_slice_get_info": [P, ctypes.POINTER(SliceInfo)],
        "ema_slice_owners": [P, P, P],
        "ema_slice_alloc_blocks": [P, I32, I32, P, P],
        "ema_slice_free_blocks": [P, P, I32],
        "ema_slice_lend": [P, I32, ctypes.POINTER(I32)],
        "ema_slice_prefetch": [P, P, P, I32, P],
        "ema_slice_migrate": [P, P, P, I32, P],
        "ema_slice_writeback": [P, P, P, I32, P],
        "ema_slice_prefetch_runs": [P, P, P, P, I32, I32, P],
        "ema_kv_append": [P, P, P, P, P, I32, I32, P],
        "ema_slice_reclaim": [P, I32, P, I64, P, ctypes.POINTER(ReclaimResult), P, I32, P, P, I32],
        "ema_paged_decode_attention": [P, P, P, P, I32, I32, I32, ctypes.c_float, P, I32, P],
        "ema_paged_decode_attention_noalloc": [P, P, P, P, I32, I32, I32, ctypes.c_float, P, I32,
                                               P],
        "ema_slice_device_errors": [P, ctypes.POINTER(I32)],
        "ema_slab_init": [P, ctypes.POINTER(SlabCfg)],
        "ema_slab_get_info": [P, ctypes.POINTER(SlabInfo), P, P],
        "ema_slab_alloc": [P, I32, P, P],
        "ema_slab_free": [P, P, I32],
        "ema_slab_block_ids": [P, P, I32, I32, I32, P],
        "ema_slab_group_runs": [P, I32, I32, P, P, P, I32, ctypes.POINTER(I32)],
        "ema_slab_prefetch_group": [P, I32, I32, I32, P],
        "ema_slab_reclaim": [P, I32, P, I64, P, ctypes.POINTER(SlabReclaimResult), P, I32, P, I32],
        "ema_kv_tables_workspace": [P, P, PSZ],
        "ema_kv_tables": [P, P, P, SZ, P],
        "ema_kv_store": [P, P, I64, P, I64, P, I32, P],
        "ema_paged_prompt_workspace": [P, I32, I32, I32, I32, PSZ],
        "ema_paged_prompt_attention": [P, P, I64, P, P, P, I32, I32, I32, I32, F32C, P, I32, P,
                                       SZ, P],
        "ema_paged_diff_workspace": [P, I32, I32, I32, PSZ],
        "ema_paged_diff_attention": [P, P, I64, P, P, I32, I32, I32, F32C, P, P, F32C, P, I32, P,
                                     SZ, P],
        "ema_paged_diff_prompt_workspace": [P, I32, I32, I32, I32, PSZ],
        "ema_paged_diff_prompt_attention": [P, P, I64, P, P, P, I32, I32, I32, I32, F32C, P, P,
                                            F32C, P, I32, P, SZ, P],
        "ema_tree_tables": [P, P, P, P, I32, I32, P, I32, P, P, P],
        "ema_paged_tree_workspace": [P, I32, I32, I32, I32, PSZ],
        "ema_paged_tree_attention": [P, P, I64, P, P, P, P, I32, I32, I32, I32, I32, F32C, P, I32,
                                     P, SZ, P],
        "ema_tree_accept": [P, P, P, P, P, P, I32, I32, I32, P, P, P, P],
        "ema_kv_compact": [P, P, P, P, P, I32, I32, I32, I32, P, P],
        "ema_sched_create": [I32, I32, I64, ctypes.POINTER(P)],
        "ema_sched_destroy": [P],
        "ema_sched_place": [P, I32, I32, I32, I64, P, ctypes.POINTER(I32)],
        "ema_sched_release": [P, I32, I32, I32],
        "ema_sched_preempted": [P, I32, I32, I64],
        "ema_sched_usage": [P, I64, P, P],
    }
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = ctypes.c_int
    lib.ema_last_error.argtypes = []
    lib.ema_last_error.restype = ctypes.c_char_p
    return lib


_lib = _load()


def _check(rc):
    if rc != OK:
        raise EmaError(rc, _lib.ema_last_error().decode())


# Per handle: host-only flag, 16-bit dtype, KV heads and blocks of both pools,
# recorded at create, so that the checks below need no library call.
_HANDLES = {}


class _Torch:
    """What the marshalling needs of torch, looked up once and on first use
    (host-only slices do not need torch): every call of a decode step passes
    here, and on small calls the host part is most of the time."""

    def __init__(self):
        import torch
        self.Tensor = torch.Tensor
        self.out_codes = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
        self.out_types = tuple(self.out_codes)
        self.i32 = (torch.int32,)
        self.f32 = (torch.float32,)
        self.i64 = (torch.int64,)
        self.kv16 = {F16: (torch.float16,), BF16: (torch.bfloat16,)}
        self.any16 = (torch.float16, torch.bfloat16, torch.int16)
        raw, dev = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream",
                                                         "_cuda_getDevice"))
        if raw and dev:
            self.stream = lambda: raw(dev())
        else:
            self.stream = lambda: torch.cuda.current_stream().cuda_stream


_TORCH = None


def _torch():
    global _TORCH
    if _TORCH is None:
        _TORCH = _Torch()
    return _TORCH


def _host_only(h):
    rec = _HANDLES.get(h)
    if rec is None:
        return slice_get_info(h)["device"] < 0
    return rec[0]


def _bad(msg):
    raise EmaError(ERR_INVAL, msg)


def _dev(t, name, dtypes, numel=0):
    """A device-array argument: a contiguous torch tensor on the GPU of one of
    ``dtypes`` with at least ``numel`` elements; returns its address. The
    kernels read whatever the pointer addresses, so a host array or a short
    tensor is refused here."""
    if not isinstance(t, _torch().Tensor) or not t.is_cuda:
        _bad(f"{name}: expected a GPU tensor, got {type(t).__name__}")
    if t.dtype not in dtypes:
        _bad(f"{name}: dtype {t.dtype} not in {dtypes}")
    if not t.is_contiguous():
        _bad(f"{name}: not contiguous")
    if t.numel() < numel:
        _bad(f"{name}: {t.numel()} elements, {numel} needed")
    return t.data_ptr()


def _i32_dev(t, name, numel=0):
    return _dev(t, name, _torch().i32, numel)


def _kv16_types(rec):
    """16-bit K/V/query types; when the handle's dtype is known, it must match."""
    T = _torch()
    return T.kv16.get(rec[1], T.any16) if rec else T.any16


def _host_ids(a, n, name):
    a = _i32_host(a)
    if len(a) < n:
        _bad(f"{name}: {len(a)} ids, {n} needed")
    return a


def _ptr(x):
    """Device address of a torch tensor, host address of a numpy array."""
    if x is None:
        return None
    if isinstance(x, np.ndarray):
        return x.ctypes.data
    return x.data_ptr()


def _i32_host(a):
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _stream(stream):
    if stream is None:
        return _torch().stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def torch_stream(stream, device=None):
    """The torch stream of what an entry point takes as one."""
    import torch
    raw = _stream(stream)
    # (an ExternalStream of 0 would be one from torch's pool)
    return torch.cuda.ExternalStream(raw, device=device) if raw else \
        torch.cuda.default_stream(device)


# ---- entry points ---------------------------------------------------------------

def slice_create(num_kv_heads, head_dim, block_size, dtype, slice_layout, local_bytes,
                 lent_bytes, host_only=False, checked=False, attn_grid=False):
    shape = KVShape(num_kv_heads, head_dim, block_size, DTYPES.get(dtype, dtype), slice_layout)
    h = ctypes.c_void_p()
    flags = ((CREATE_HOST_ONLY if host_only else 0) | (CREATE_CHECKED if checked else 0)
             | (CREATE_ATTN_GRID if attn_grid else 0))
    _check(_lib.ema_slice_create(ctypes.byref(shape), int(local_bytes), int(lent_bytes), flags,
                                 ctypes.byref(h)))
    bb = 2 * shape.block_size * shape.num_kv_heads * shape.head_dim * 2
    _HANDLES[h.value] = (bool(host_only), shape.dtype, int(num_kv_heads),
                         int(local_bytes) // bb + int(lent_bytes) // bb)
    return h.value


def slice_destroy(h):
    _check(_lib.ema_slice_destroy(h))
    _HANDLES.pop(h, None)


def slice_get_info(h):
    info = SliceInfo()
    _check(_lib.ema_slice_get_info(h, ctypes.byref(info)))
    return {k: getattr(info, k) for k, _ in SliceInfo._fields_}


def slice_owners(h):
    info = slice_get_info(h)
    own_l = np.empty(info["n_local"], dtype=np.int32)
    own_s = np.empty(info["n_slice"], dtype=np.int32)
    _check(_lib.ema_slice_owners(h, own_l.ctypes.data, own_s.ctypes.data))
    return own_l, own_s, info["lim"]


def slice_alloc_blocks(h, pool, owners):
    owners = _i32_host(owners)
    out = np.empty(len(owners), dtype=np.int32)
    _check(_lib.ema_slice_alloc_blocks(h, pool, len(owners), owners.ctypes.data, out.ctypes.data))
    return out


def slice_free_blocks(h, ids):
    ids = _i32_host(ids)
    _check(_lib.ema_slice_free_blocks(h, ids.ctypes.data, len(ids)))


def slice_lend(h, n_blocks):
    added = ctypes.c_int32()
    _check(_lib.ema_slice_lend(h, int(n_blocks), ctypes.byref(added)))
    return added.value


def _copy_call(fn, h, src, dst, n, stream):
    n = len(src) if n is None else int(n)
    if _host_only(h):
        src, dst = _host_ids(src, n, "source ids"), _host_ids(dst, n, "destination ids")
        _check(fn(h, _ptr(src), _ptr(dst), n, None))
        return
    _check(fn(h, _i32_dev(src, "source ids", n), _i32_dev(dst, "destination ids", n), n,
              _stream(stream)))


def slice_prefetch(h, block_ids, dst_block_table, n=None, stream=None):
    """block_ids, dst_block_table: int32 device tensors (numpy arrays for a
    host-only slice)."""
    _copy_call(_lib.ema_slice_prefetch, h, block_ids, dst_block_table, n, stream)


def slice_migrate(h, src_ids, dst_ids, n=None, stream=None):
    _copy_call(_lib.ema_slice_migrate, h, src_ids, dst_ids, n, stream)


def slice_prefetch_runs(h, src_first, dst_first, run_blocks, engine=0, stream=None):
    """Contiguous runs (host int arrays); engine ENGINE_KERNEL or ENGINE_DMA."""
    src_first, dst_first, run_blocks = (_i32_host(a) for a in (src_first, dst_first, run_blocks))
    info_host = _host_only(h)
    _check(_lib.ema_slice_prefetch_runs(h, src_first.ctypes.data, dst_first.ctypes.data,
                                        run_blocks.ctypes.data, len(run_blocks), int(engine),
                                        None if info_host else _stream(stream)))


def slice_writeback(h, staging_ids, slice_ids, n=None, stream=None):
    """staging_ids, slice_ids: int32 device tensors (numpy arrays for a
    host-only slice)."""
    _copy_call(_lib.ema_slice_writeback, h, staging_ids, slice_ids, n, stream)


def kv_append(h, k_new, v_new, block_table, seq_lens, stream=None):
    """k_new, v_new [B][Hkv][D] (16-bit), block_table int32 [B][max_blocks],
    seq_lens int32 [B] counting the new token: device tensors (numpy arrays
    for a host-only slice)."""
    shape = block_table.shape
    B = int(shape[0])
    max_blocks = int(shape[1]) if len(shape) == 2 else 0
    if _host_only(h):
        block_table, seq_lens = _i32_host(block_table), _i32_host(seq_lens)
        _check(_lib.ema_kv_append(h, _ptr(k_new), _ptr(v_new), _ptr(block_table), _ptr(seq_lens),
                                  B, max_blocks, None))
        return
    rec = _HANDLES.get(h)
    row = rec[2] * 128 if rec else 0          # K/V elements per sequence
    kv16 = _kv16_types(rec)
    table = _i32_dev(block_table, "block_table", B * max_blocks)
    lens = _i32_dev(seq_lens, "seq_lens", B)
    _check(_lib.ema_kv_append(h, _dev(k_new, "k_new", kv16, B * row),
                              _dev(v_new, "v_new", kv16, B * row), table, lens, B, max_blocks,
                              _stream(stream)))


def slice_reclaim(h, n_blocks, canon_tables=None, stream=None, caps=None):
    """canon_tables: int32 device tensor rewritten in place (None for none).
    Returns the result counts, the victims (list) and the copies made
    ("moves": int64 array [moved][2] of (source, destination) unified ids)."""
    rec = _HANDLES.get(h)
    if rec is None:
        info = slice_get_info(h)
        rec = (info["device"] < 0, None, 0, info["n_local"] + info["n_slice"])
    cap = int(caps) if caps is not None else rec[3]
    res = ReclaimResult()
    victims = np.empty(max(cap, 1), dtype=np.int32)
    msrc = np.empty(max(cap, 1), dtype=np.int32)
    mdst = np.empty(max(cap, 1), dtype=np.int32)
    host_only = rec[0]
    if canon_tables is not None and not host_only:
        _i32_dev(canon_tables, "canon_tables")
    n_entries = 0 if canon_tables is None else canon_tables.numel()
    _check(_lib.ema_slice_reclaim(h, int(n_blocks), _ptr(canon_tables), n_entries,
                                  None if host_only else _stream(stream), ctypes.byref(res),
                                  victims.ctypes.data, cap, msrc.ctypes.data, mdst.ctypes.data,
                                  cap))
    m = min(res.moved, cap)
    return {"reclaimed": res.reclaimed, "moved": res.moved, "written_back": res.written_back,
            "victims": victims[:min(res.n_victims, cap)].tolist(), "lim": res.lim,
            "moves": np.stack([msrc[:m], mdst[:m]], axis=1).astype(np.int64)}


def _attention_call(fn, h, q, block_table, seq_lens, out, scale, stream):
    T = _torch()
    shape, tshape = q.shape, block_table.shape
    B, Hq = int(shape[0]), int(shape[1])
    max_blocks = int(tshape[1]) if len(tshape) == 2 else 0
    code = T.out_codes.get(out.dtype)
    if code is None:
        _bad(f"out: dtype {out.dtype} not in {T.out_types}")
    rec = _HANDLES.get(h)
    if rec[0] if rec else _host_only(h):
        args = _ptr(q), _ptr(block_table), _ptr(seq_lens), _ptr(out)
    else:
        args = (_dev(q, "q", _kv16_types(rec), B * Hq * 128),
                _i32_dev(block_table, "block_table", B * max_blocks),
                _i32_dev(seq_lens, "seq_lens", B), _dev(out, "out", T.out_types, B * Hq * 128))
    _check(fn(h, args[0], args[1], args[2], B, Hq, max_blocks, float(scale), args[3], code,
              _stream(stream)))


def paged_decode_attention(h, q, block_table, seq_lens, out, scale=0.0, stream=None):
    """q [B][Hq][D] (16-bit), block_table int32 [B][max_blocks], seq_lens int32
    [B], out [B][Hq][D] of float32, float16 or bfloat16 (the output type is
    the tensor's): device tensors."""
    _attention_call(_lib.ema_paged_decode_attention, h, q, block_table, seq_lens, out, scale,
                    stream)


def paged_decode_attention_noalloc(h, q, block_table, seq_lens, out, scale=0.0, stream=None):
    """The same as paged_decode_attention, in the library's fixed per-GPU
    workspace: for callers that cannot allocate (see the C header)."""
    _attention_call(_lib.ema_paged_decode_attention_noalloc, h, q, block_table, seq_lens, out,
                    scale, stream)


def slice_device_errors(h):
    c = ctypes.c_int32()
    _check(_lib.ema_slice_device_errors(h, ctypes.byref(c)))
    return c.value


# ---- prompts and differential attention (include/ema_ops.h) --------------------------

def _scratch(nbytes, workspace, stream, device):
    """(tensor, address, bytes) of a call's workspace: the caller's, or one from
    torch's allocator."""
    if workspace is None:
        if nbytes == 0:
            return None, None, 0
        import torch
        if stream == _torch().stream():
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
        else:                             # memory that nothing on another stream still uses
            with torch.cuda.stream(torch_stream(stream, device)):
                workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
    n = workspace.numel() * workspace.element_size()
    if n < nbytes:
        _bad(f"workspace: {n} bytes, {nbytes} needed")
    return workspace, _dev(workspace, "workspace", (workspace.dtype,)), n


def _i32_exact(t, name, host, shape):
    """Address of an int32 array of exactly this shape."""
    if t.shape != shape:
        _bad(f"{name}: shape {tuple(t.shape)}, expected {shape}")
    if host:
        if not isinstance(t, np.ndarray) or t.dtype != np.int32 or not t.flags.c_contiguous:
            _bad(f"{name}: expected a contiguous int32 numpy array")
        return t.ctypes.data
    return _dev(t, name, _torch().i32)


def _tables_args(host, block_ids, seq_lens, new_lens, block_table, slot_map, query_start,
                 canon_table, staging, prefetch, writeback):
    try:
        L, B, max_blocks = block_table.shape
        (_, n_ids), (_, n_slots) = block_ids.shape, slot_map.shape
    except ValueError:
        _bad("expected block_table [L][B][max_blocks], block_ids [L][n_ids], slot_map [L][n_slots]")
    addr = [_i32_exact(block_ids, "block_ids", host, (L, n_ids)),
            _i32_exact(seq_lens, "seq_lens", host, (B,)),
            _i32_exact(new_lens, "new_lens", host, (B,)), None,
            None if canon_table is None else
            _i32_exact(canon_table, "canon_table", host, (L, B, max_blocks)),
            _i32_exact(block_table, "block_table", host, (L, B, max_blocks)),
            _i32_exact(query_start, "query_start", host, (B + 1,)),
            _i32_exact(slot_map, "slot_map", host, (L, n_slots))]
    slots = stage_n = cap = 0
    if staging is not None:
        if prefetch is None or writeback is None:
            _bad("staging needs the prefetch and writeback lists")
        try:
            slots, stage_n = staging.shape
            _, _, _ = prefetch
            to_write, _, _ = writeback
            _, cap = to_write.shape
        except ValueError:
            _bad("expected staging [slots][stage_n] and lists (source [L][n], destination, count)")
        addr[3] = _i32_exact(staging, "staging", host, (slots, stage_n))
        for kind, (src, dst, count), n in (("prefetch", prefetch, stage_n),
                                           ("writeback", writeback, cap)):
            addr += [_i32_exact(src, kind, host, (L, n)), _i32_exact(dst, kind, host, (L, n)),
                     _i32_exact(count, kind, host, (L,))]
    else:
        addr += [None] * 6
    return KVTablesArgs(*addr, L, B, max_blocks, n_ids, n_slots, slots, stage_n, cap)


def kv_tables_workspace(h, args):
    """Bytes of workspace for a KVTablesArgs."""
    n = ctypes.c_size_t()
    _check(_lib.ema_kv_tables_workspace(h, ctypes.byref(args), ctypes.byref(n)))
    return n.value


def kv_tables(h, block_ids, seq_lens, new_lens, block_table, slot_map, query_start,
              canon_table=None, staging=None, prefetch=None, writeback=None, workspace=None,
              stream=None):
    """The tables of a step for all layers, from the requests' lengths: block_ids
    [L][n_ids], seq_lens and new_lens [B] in; block_table [L][B][max_blocks],
    slot_map [L][n_slots], query_start [B + 1] and, if given, canon_table out.
    With ``staging`` [slots][stage_n] slice blocks are named by their staged copies,
    and ``prefetch`` (src [L][stage_n], dst, count [L]) and ``writeback`` (src
    [L][cap], dst, count [L]) are written. int32 device tensors (numpy arrays for
    a host-only slice, which only validates)."""
    rec = _HANDLES.get(h)
    host = rec[0] if rec else _host_only(h)
    a = _tables_args(host, block_ids, seq_lens, new_lens, block_table, slot_map, query_start,
                     canon_table, staging, prefetch, writeback)
    if host:
        _check(_lib.ema_kv_tables(h, ctypes.byref(a), None, 0, None))
        return
    st = _stream(stream)
    size = 0 if staging is None else kv_tables_workspace(h, a)
    ws, p, n = _scratch(size, workspace, st, block_table.device)
    _check(_lib.ema_kv_tables(h, ctypes.byref(a), p, n, st))


def _rows16(t, name, types, heads):
    """(address, elements between tokens) of a 16-bit GPU tensor [T][heads][128]
    whose tokens may lie apart."""
    if not isinstance(t, _torch().Tensor) or not t.is_cuda:
        _bad(f"{name}: expected a GPU tensor, got {type(t).__name__}")
    if t.dtype not in types:
        _bad(f"{name}: dtype {t.dtype} not in {types}")
    shape = t.shape
    if len(shape) != 3 or shape[2] != 128 or (heads and shape[1] != heads):
        _bad(f"{name}: shape {tuple(shape)}, expected [tokens][{heads or 'heads'}][128]")
    row = shape[1] * 128
    if t.is_contiguous():
        return t.data_ptr(), row
    stride = t.stride()
    if stride[2] != 1 or (shape[1] > 1 and stride[1] != 128):
        _bad(f"{name}: a token's heads are not contiguous")
    return t.data_ptr(), stride[0] if shape[0] > 1 else row


def kv_store(h, k_new, v_new, slot_map, stream=None):
    """k_new, v_new [T][Hkv][128] (16-bit; a token's heads contiguous, tokens any
    multiple of 8 elements apart), slot_map int32 [T] (-1: not stored): device
    tensors (a host-only slice takes slot_map as a numpy array and validates it)."""
    if _host_only(h):
        slots = _i32_host(slot_map)
        row = int(_HANDLES[h][2]) * 128 if h in _HANDLES else 64 * 128
        _check(_lib.ema_kv_store(h, None, row, None, row, slots.ctypes.data, len(slots), None))
        return
    rec = _HANDLES.get(h)
    heads, types = rec[2] if rec else 0, _kv16_types(rec)
    k, ks = _rows16(k_new, "k_new", types, heads)
    v, vs = _rows16(v_new, "v_new", types, heads)
    T = k_new.shape[0]
    if v_new.shape != k_new.shape:
        _bad(f"v_new: shape {tuple(v_new.shape)}, k_new has {tuple(k_new.shape)}")
    if slot_map.numel() != T:
        _bad(f"slot_map: {slot_map.numel()} slots, {T} tokens")
    _check(_lib.ema_kv_store(h, k, ks, v, vs, _i32_dev(slot_map, "slot_map", T), T,
                             _stream(stream)))


def _attention_op(h, fn, size, maps, q, query_start, block_table, seq_lens, out, scale, lam,
                  norm_weight, norm_eps, full_weights, workspace, stream, mask=None):
    T = _torch()
    try:
        rows, Hq, _ = q.shape
        B, max_blocks = block_table.shape
    except ValueError:
        _bad("expected q [tokens][heads][128] and block_table [batch][max_blocks]")
    extra = () if maps == 1 else (None, None, float(norm_eps))
    sizes = (rows, B, Hq, max_blocks) if query_start is not None else (B, Hq, max_blocks)
    if query_start is None and rows != B:
        _bad(f"q: {rows} rows, {B} sequences")
    rec = _HANDLES.get(h)
    if rec[0] if rec else _host_only(h):
        table, lens = _i32_host(block_table), _i32_host(seq_lens)
        starts = () if query_start is None else (_i32_host(query_start).ctypes.data,)
        masks = () if mask is None else (None, _mask_shape(mask, rows))
        _check(fn(h, None, Hq * 128, *starts, table.ctypes.data, lens.ctypes.data, *masks, *sizes,
                  float(scale), *extra, None, F32, None, 0, None))
        return
    code = T.out_codes.get(out.dtype)
    if code is None:
        _bad(f"out: dtype {out.dtype} not in {T.out_types}")
    qp, qs = _rows16(q, "q", _kv16_types(rec), 0)
    starts = () if query_start is None else (_i32_dev(query_start, "query_start", B + 1),)
    table = _i32_dev(block_table, "block_table", B * max_blocks)
    lens = _i32_dev(seq_lens, "seq_lens", B)
    masks = () if mask is None else _mask_words(mask, rows)
    if maps == 2:
        extra = (_dev(lam, "lam", T.f32, Hq // 2),
                 None if norm_weight is None else _dev(norm_weight, "norm_weight", T.f32, 256),
                 float(norm_eps))
    dst = _dev(out, "out", T.out_types, rows * Hq * 128)
    if full_weights:
        code |= FULL_WEIGHTS
    st = _stream(stream)
    n = ctypes.c_size_t()
    _check(size(h, *sizes, ctypes.byref(n)))
    ws, p, nbytes = _scratch(n.value, workspace, st, q.device)
    _check(fn(h, qp, qs, *starts, table, lens, *masks, *sizes, float(scale), *extra, dst, code, p,
              nbytes, st))


def _size_call(fn, *args):
    n = ctypes.c_size_t()
    _check(fn(*args, ctypes.byref(n)))
    return n.value


def paged_prompt_workspace(h, tokens, batch, num_q_heads, max_blocks):
    return _size_call(_lib.ema_paged_prompt_workspace, h, tokens, batch, num_q_heads, max_blocks)


def paged_diff_workspace(h, batch, num_q_heads, max_blocks):
    return _size_call(_lib.ema_paged_diff_workspace, h, batch, num_q_heads, max_blocks)


def paged_diff_prompt_workspace(h, tokens, batch, num_q_heads, max_blocks):
    return _size_call(_lib.ema_paged_diff_prompt_workspace, h, tokens, batch, num_q_heads,
                      max_blocks)


def paged_prompt_attention(h, q, query_start, block_table, seq_lens, out, scale=0.0,
                           workspace=None, stream=None, full_weights=False):
    """Causal attention of prompt chunks: q [T][Hq][128] (16-bit, tokens any multiple
    of 8 elements apart), query_start int32 [B + 1], block_table int32
    [B][max_blocks], seq_lens int32 [B], out [T][Hq][128] of float32, float16 or
    bfloat16. A 16-bit out rounds the softmax weights once, or with ``full_weights`` keeps
    them to 32-bit accuracy as a float32 out does, in its time. Without ``workspace`` (a byte
    tensor of paged_prompt_workspace bytes) the call takes one from torch's allocator."""
    _attention_op(h, _lib.ema_paged_prompt_attention, _lib.ema_paged_prompt_workspace, 1, q,
                  query_start, block_table, seq_lens, out, scale, None, None, 0.0, full_weights,
                  workspace, stream)


def paged_diff_attention(h, q, block_table, seq_lens, lam, out, scale=0.0, norm_weight=None,
                         norm_eps=0.0, workspace=None, stream=None, full_weights=False):
    """Differential attention of one token per sequence: q [B][Hq][128], lam float32
    [Hq / 2], out [B][Hq / 2][256]; with norm_weight (float32 [256]) each output
    row is divided by its root mean square and multiplied by it. full_weights as in
    paged_prompt_attention (without it a bfloat16 out has weights of 16 bits)."""
    _attention_op(h, _lib.ema_paged_diff_attention, _lib.ema_paged_diff_workspace, 2, q, None,
                  block_table, seq_lens, out, scale, lam, norm_weight, norm_eps, full_weights,
                  workspace, stream)


def paged_diff_prompt_attention(h, q, query_start, block_table, seq_lens, lam, out, scale=0.0,
                                norm_weight=None, norm_eps=0.0, workspace=None, stream=None,
                                full_weights=False):
    """Differential attention of prompt chunks: rows as in paged_prompt_attention,
    heads, lam and norm as in paged_diff_attention; out [T][Hq / 2][256]."""
    _attention_op(h, _lib.ema_paged_diff_prompt_attention, _lib.ema_paged_diff_prompt_workspace, 2,
                  q, query_start, block_table, seq_lens, out, scale, lam, norm_weight, norm_eps,
                  full_weights, workspace, stream)


# ---- trees of drafted tokens (include/ema_tree.h) -------------------------------------

def _i32_args(host, arrays):
    """Addresses of int32 arrays (name, array or None, elements it must have)."""
    if not host:
        T, addr = _torch(), []
        Tensor, (int32,) = T.Tensor, T.i32
        for name, t, n in arrays:
            if t is None:
                addr.append(None)
            elif type(t) is Tensor and t.is_cuda and t.dtype is int32 and t.numel() == n and \
                    t.is_contiguous():
                addr.append(t.data_ptr())
            else:
                addr.append(_dev(t, name, T.i32))
                if t.numel() != n:
                    _bad(f"{name}: {t.numel()} elements, expected {n}")
        return addr
    addr = []
    for name, t, n in arrays:
        if t is None:
            addr.append(None)
        else:
            if not isinstance(t, np.ndarray) or t.dtype != np.int32 or not t.flags.c_contiguous:
                _bad(f"{name}: expected a contiguous int32 numpy array")
            if t.size != n:
                _bad(f"{name}: {t.size} elements, expected {n}")
            addr.append(t.ctypes.data)
    return addr


def _rows_and_batch(parents, query_start):
    try:
        (rows,), (B,) = parents.shape, query_start.shape
    except ValueError:
        _bad("expected parents [tokens] and query_start [batch + 1]")
    if B < 1:
        _bad("query_start: empty")
    return rows, B - 1


def _mask_shape(mask, rows):
    """Words of the masks of `rows` rows."""
    shape = mask.shape
    if len(shape) != 2 or shape[0] != rows:
        _bad(f"mask: shape {tuple(shape)}, expected [{rows}][words]")
    return shape[1]


def _mask_words(mask, rows):
    """(address, words) of the masks of `rows` rows."""
    words = _mask_shape(mask, rows)
    return _dev(mask, "mask", _torch().i64), words


def tree_tables(h, parents, query_start, seq_lens, mask, positions=None, base=None, stream=None):
    """What the nodes of drafted trees attend and where they stand: parents int32 [T] (a
    node's parent within its request, -1: a root), query_start int32 [B + 1], seq_lens int32
    [B] in; mask int64 [T][words] (64 nodes a word), positions int32 [T] and base int32 [B]
    (tokens before the tree) out. Device tensors (numpy arrays for a host-only slice,
    which only validates)."""
    rows, B = _rows_and_batch(parents, query_start)
    rec = _HANDLES.get(h)
    host = rec[0] if rec else _host_only(h)
    addr = _i32_args(host, (("parents", parents, rows), ("query_start", query_start, B + 1),
                            ("seq_lens", seq_lens, B), ("positions", positions, rows),
                            ("base", base, B)))
    if host:
        at, words, st = None, _mask_shape(mask, rows), None
    else:
        (at, words), st = _mask_words(mask, rows), _stream(stream)
    _check(_lib.ema_tree_tables(h, *addr[:3], rows, B, at, words, *addr[3:], st))


def paged_tree_workspace(h, tokens, batch, num_q_heads, max_blocks):
    return _size_call(_lib.ema_paged_tree_workspace, h, tokens, batch, num_q_heads, max_blocks)


def paged_tree_attention(h, q, query_start, block_table, seq_lens, mask, out, scale=0.0,
                         workspace=None, stream=None, full_weights=False):
    """Attention of drafted nodes: mask int64 [T][words] says which of its request's nodes a
    row attends beside all tokens before them (bit j: the node in the j-th of the request's
    rows, which are its last tokens); the other arrays as in paged_prompt_attention."""
    if mask is None:
        _bad("mask: missing")
    _attention_op(h, _lib.ema_paged_tree_attention, _lib.ema_paged_tree_workspace, 1, q,
                  query_start, block_table, seq_lens, out, scale, None, None, 0.0, full_weights,
                  workspace, stream, mask)


def tree_accept(h, parents, query_start, drafted, choice, path, n_path, next_token,
                root_choice=None, stream=None):
    """The path of each tree that the model's choices confirm: parents, drafted (the nodes'
    tokens), choice (the model's after them) int32 [T], query_start [B + 1], root_choice
    int32 [B] (the model's choice before the tree; None: node 0 is accepted as it is) in; path
    int32 [B][cap] (-1 behind the path), n_path and next_token int32 [B] out."""
    rows, B = _rows_and_batch(parents, query_start)
    shape = path.shape
    if len(shape) != 2 or shape[0] != B:
        _bad(f"path: shape {tuple(shape)}, expected [{B}][cap]")
    rec = _HANDLES.get(h)
    host = rec[0] if rec else _host_only(h)
    addr = _i32_args(host, (("parents", parents, rows), ("query_start", query_start, B + 1),
                            ("drafted", drafted, rows), ("choice", choice, rows),
                            ("root_choice", root_choice, B), ("path", path, B * shape[1]),
                            ("n_path", n_path, B), ("next_token", next_token, B)))
    _check(_lib.ema_tree_accept(h, *addr[:5], rows, B, shape[1], *addr[5:],
                                None if host else _stream(stream)))


def kv_compact(h, block_table, base, keep, n_keep, new_lens=None, stream=None):
    """Moves kept tokens together, in all layers and in place: token base[b] + k becomes what
    token base[b] + keep[b][k] was, k < n_keep[b]; new_lens[b] = base[b] + n_keep[b].
    block_table int32 [L][B][max_blocks] (unified ids), base, n_keep, new_lens int32
    [B], keep int32 [B][cap], ascending."""
    try:
        (L, B, width), (_, cap) = block_table.shape, keep.shape
    except ValueError:
        _bad("expected block_table [L][B][max_blocks] and keep [B][cap]")
    rec = _HANDLES.get(h)
    host = rec[0] if rec else _host_only(h)
    addr = _i32_args(host, (("block_table", block_table, L * B * width), ("base", base, B),
                            ("keep", keep, B * cap), ("n_keep", n_keep, B),
                            ("new_lens", new_lens, B)))
    _check(_lib.ema_kv_compact(h, *addr[:4], L, B, width, cap, addr[4],
                               None if host else _stream(stream)))


# ---- slab management of the slice --------------------------------------------------

def slab_init(h, layers, slab_blocks, group, layout=SLAB_GROUP_MAJOR):
    cfg = SlabCfg(int(layers), int(slab_blocks), int(group), int(layout))
    _check(_lib.ema_slab_init(h, ctypes.byref(cfg)))


def slab_get_info(h):
    """Shape and state: dict with n_slabs, layers, slab_blocks, group, layout,
    borrowed, slab_tag (int32 [n_slabs]) and pos_owner (int32 [n_slabs * S])."""
    info = SlabInfo()
    _check(_lib.ema_slab_get_info(h, ctypes.byref(info), None, None))
    tag = np.empty(info.n_slabs, dtype=np.int32)
    own = np.empty(info.n_slabs * info.slab_blocks, dtype=np.int32)
    _check(_lib.ema_slab_get_info(h, ctypes.byref(info), tag.ctypes.data, own.ctypes.data))
    d = {k: getattr(info, k) for k, _ in SlabInfo._fields_}
    d["slab_tag"], d["pos_owner"] = tag, own
    return d


def slab_alloc(h, owners):
    owners = _i32_host(owners)
    out = np.empty(len(owners), dtype=np.int32)
    _check(_lib.ema_slab_alloc(h, len(owners), owners.ctypes.data, out.ctypes.data))
    return out


def slab_free(h, positions):
    positions = _i32_host(positions)
    _check(_lib.ema_slab_free(h, positions.ctypes.data, len(positions)))


def slab_block_ids(h, positions, layer, staging_first=-1):
    """Unified ids of `layer`'s blocks at the positions (slice blocks, or
    their staged copies when staging_first >= 0)."""
    positions = _i32_host(positions)
    out = np.empty(len(positions), dtype=np.int32)
    _check(_lib.ema_slab_block_ids(h, positions.ctypes.data, len(positions), int(layer),
                                   int(staging_first), out.ctypes.data))
    return out


def slab_group_runs(h, group, staging_first):
    """(src_first, dst_first, run_blocks) int32 arrays of the group's swap."""
    n = ctypes.c_int32()
    _check(_lib.ema_slab_group_runs(h, int(group), int(staging_first), None, None, None, 0,
                                    ctypes.byref(n)))
    a, b, c = (np.empty(max(n.value, 1), dtype=np.int32) for _ in range(3))
    _check(_lib.ema_slab_group_runs(h, int(group), int(staging_first), a.ctypes.data,
                                    b.ctypes.data, c.ctypes.data, n.value, ctypes.byref(n)))
    return a[:n.value], b[:n.value], c[:n.value]


def slab_prefetch_group(h, group, staging_first, engine=ENGINE_KERNEL, stream=None):
    _check(_lib.ema_slab_prefetch_group(h, int(group), int(staging_first), int(engine),
                                        None if _host_only(h) else _stream(stream)))


def slab_reclaim(h, n_slabs, canon_tables=None, stream=None):
    """Returns reclaimed, n_victims, released counts plus the slabs taken and
    the victims (lists)."""
    info = slab_get_info(h)
    res = SlabReclaimResult()
    slabs = np.empty(max(info["n_slabs"], 1), dtype=np.int32)
    cap = int(info["n_slabs"] * info["slab_blocks"] + 1)
    victims = np.empty(cap, dtype=np.int32)
    host_only = _host_only(h)
    if canon_tables is not None and not host_only:
        _i32_dev(canon_tables, "canon_tables")
    n_entries = 0 if canon_tables is None else canon_tables.numel()
    _check(_lib.ema_slab_reclaim(h, int(n_slabs), _ptr(canon_tables), n_entries,
                                 None if host_only else _stream(stream), ctypes.byref(res),
                                 slabs.ctypes.data, len(slabs), victims.ctypes.data, cap))
    return {"reclaimed": res.reclaimed, "released": res.released,
            "slabs": slabs[:res.reclaimed].tolist(),
            "victims": victims[:min(res.n_victims, cap)].tolist()}


# ---- slice scheduling across GPUs (host policy) -------------------------------------

def sched_create(n_gpus, slice_units, cap_window=0):
    h = ctypes.c_void_p()
    _check(_lib.ema_sched_create(int(n_gpus), int(slice_units), int(cap_window), ctypes.byref(h)))
    return h.value


def sched_destroy(s):
    _check(_lib.ema_sched_destroy(s))


def sched_place(s, gpu, req, n, t=0):
    """Peers of the slices the n units went to (-1: refused)."""
    peers = np.empty(max(int(n), 1), dtype=np.int32)
    placed = ctypes.c_int32()
    _check(_lib.ema_sched_place(s, int(gpu), int(req), int(n), int(t), peers.ctypes.data,
                                ctypes.byref(placed)))
    return peers[:int(n)].tolist()


def sched_release(s, gpu, req, n):
    _check(_lib.ema_sched_release(s, int(gpu), int(req), int(n)))


def sched_preempted(s, gpu, peer, t):
    _check(_lib.ema_sched_preempted(s, int(gpu), int(peer), int(t)))


def sched_usage(s, m, t=0):
    """(use, cap) as int arrays [m][m]; cap -1 where none is active."""
    use = np.empty(m * m, dtype=np.int32)
    cap = np.empty(m * m, dtype=np.int32)
    _check(_lib.ema_sched_usage(s, int(t), use.ctypes.data, cap.ctypes.data))
    return use.reshape(m, m), cap.reshape(m, m)


class Scheduler:
    """Greedy-Least-Loaded placement over the slices of n_gpus GPUs, with
    bursty preemption caps (the sched_* calls on one handle)."""

    def __init__(self, n_gpus, slice_units, cap_window=0):
        self.m = int(n_gpus)
        self.h = sched_create(n_gpus, slice_units, cap_window)

    def place(self, gpu, req, n, t=0):
        return sched_place(self.h, gpu, req, n, t)

    def release(self, gpu, req, n):
        sched_release(self.h, gpu, req, n)

    def preempted(self, gpu, peer, t):
        sched_preempted(self.h, gpu, peer, t)

    def usage(self, t=0):
        return sched_usage(self.h, self.m, t)

    def close(self):
        if self.h:
            sched_destroy(self.h)
            self.h = None


# ---- plumbing: library-owned pools as torch tensors ---------------------------------

class _DeviceBuffer:
    def __init__(self, ptr, nbytes):
        self.__cuda_array_interface__ = {"shape": (int(nbytes),), "typestr": "|u1",
                                         "data": (int(ptr), False), "version": 3,
                                         "strides": None}


def pool_view(h, pool):
    """uint8 torch tensor [n_blocks][block_bytes] aliasing a library pool.
    Valid until slice_destroy(h)."""
    import torch
    info = slice_get_info(h)
    n = info["n_local"] if pool == POOL_LOCAL else info["n_slice"]
    base = info["local_base"] if pool == POOL_LOCAL else info["slice_base"]
    if n == 0 or not base:
        return torch.empty((0, info["block_bytes"]), dtype=torch.uint8, device="cuda")
    t = torch.as_tensor(_DeviceBuffer(base, n * info["block_bytes"]), device="cuda")
    return t.view(n, info["block_bytes"])


def last_error():
    return _lib.ema_last_error().decode()
