"""ctypes binding of libburstattn's C ABI (include/burst_attn.h, burst_lm_head.h and burst_attn_cache.h).

Argument marshalling only: every function here has the name of the C entry point
it calls and does nothing but describe torch tensors as (pointer, strides) and
pass the current HIP stream.  There is no fallback: if the shared library has
not been built, importing this module raises.
"""
import ctypes as C
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("BURST_LIB_PATH", os.path.join(_HERE, "libburstattn.so"))   # override: another build

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} not found: build it first (python -m paper_2509_19836_amd.build, or "
        "__graft_entry__.build()); libburstattn has no CPU or PyTorch fallback")
_lib = C.CDLL(LIB_PATH)

BURST_OK, BURST_ERR_INVALID_ARG, BURST_ERR_UNSUPPORTED, BURST_ERR_HIP, BURST_ERR_SCRATCH = 0, -1, -2, -3, -4
BURST_BF16, BURST_F32, BURST_F8E4M3 = 0, 1, 2
BURST_MASK_FULL, BURST_MASK_CAUSAL = 0, 1
BURST_ACC_DQ, BURST_ACC_DK, BURST_ACC_DV = 1, 2, 4
BURST_MAX_STEPS = 1024
BURST_TREE_MAX_TOKENS, BURST_CACHE_MAX_LAYERS, BURST_SCORES_MAX_TOP = 64, 1024, 64
BURST_KERNEL_DQ, BURST_KERNEL_DKDV, BURST_KERNEL_DEALT, BURST_KERNEL_SHARED_CU, BURST_KERNEL_KEY_TILES_64 = 1, 2, 4, 8, 16


class burst_shape_t(C.Structure):
    _fields_ = [("batch", C.c_int32), ("q_heads", C.c_int32), ("kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("sq", C.c_int64), ("sk", C.c_int64), ("scale", C.c_float)]


class burst_tensor_t(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("dtype", C.c_int32), ("_pad", C.c_int32),
                ("stride_b", C.c_int64), ("stride_s", C.c_int64), ("stride_h", C.c_int64)]


class burst_rowvec_t(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("stride_b", C.c_int64), ("stride_h", C.c_int64)]


class burst_mask_t(C.Structure):
    _fields_ = [("mode", C.c_int32), ("q_nseg", C.c_int32), ("k_nseg", C.c_int32), ("_pad", C.c_int32),
                ("q_seg_pos", C.c_int64 * 2), ("k_seg_pos", C.c_int64 * 2),
                ("q_seg_len", C.c_int64), ("k_seg_len", C.c_int64), ("pos_stride", C.c_int64),
                ("window", C.c_int64), ("block_mask", C.c_void_p),
                ("q_block_rows", C.c_int64), ("k_block_rows", C.c_int64), ("block_pitch", C.c_int64)]


_P = C.POINTER
_lib.burst_attn_step_fwd.restype = C.c_int
_lib.burst_attn_step_fwd.argtypes = [_P(burst_shape_t), _P(burst_mask_t)] + [_P(burst_tensor_t)] * 3 + [
    _P(burst_tensor_t), _P(burst_rowvec_t), _P(burst_tensor_t), _P(burst_rowvec_t), C.c_void_p]
_lib.burst_attn_lse_merge.restype = C.c_int
_lib.burst_attn_lse_merge.argtypes = [_P(burst_shape_t), _P(burst_tensor_t), _P(burst_rowvec_t),
                                      _P(burst_tensor_t), _P(burst_rowvec_t), _P(burst_tensor_t), C.c_void_p]
_lib.burst_attn_preprocess_bwd.restype = C.c_int
_lib.burst_attn_preprocess_bwd.argtypes = [_P(burst_shape_t), _P(burst_tensor_t), _P(burst_tensor_t),
                                           _P(burst_rowvec_t), C.c_void_p]
_lib.burst_attn_step_bwd.restype = C.c_int
_lib.burst_attn_step_bwd.argtypes = [_P(burst_shape_t), _P(burst_mask_t)] + [_P(burst_tensor_t)] * 4 + [
    _P(burst_rowvec_t)] * 2 + [_P(burst_tensor_t)] * 3 + [C.c_int32, C.c_void_p]
_lib.burst_attn_steps_fwd.restype = C.c_int
# (arrays of structs go in as the bytes they consist of)
_lib.burst_attn_steps_fwd.argtypes = [C.c_int32, C.c_char_p, _P(burst_mask_t), _P(burst_tensor_t), C.c_char_p, C.c_char_p,
                                      _P(burst_tensor_t), _P(burst_rowvec_t), C.c_void_p]
_lib.burst_attn_steps_bwd.restype = C.c_int
_lib.burst_attn_steps_bwd.argtypes = [C.c_int32, C.c_char_p, _P(burst_mask_t), _P(burst_tensor_t), C.c_char_p, C.c_char_p,
                                      _P(burst_tensor_t), _P(burst_rowvec_t), _P(burst_rowvec_t), _P(burst_tensor_t),
                                      C.c_char_p, C.c_char_p, C.c_int32, C.c_void_p]
_lib.burst_attn_fill_ring_masks.restype = C.c_int
_lib.burst_attn_fill_ring_masks.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int64, C.c_int64, C.c_int64, _P(burst_mask_t)]
for _name in ("zigzag", "contiguous", "striped"):
    _f = getattr(_lib, f"burst_attn_fill_{_name}_mask")
    _f.restype = C.c_int
    _f.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int64, C.c_int32, _P(burst_mask_t)]
_lib.burst_attn_fill_block_striped_mask.restype = C.c_int
_lib.burst_attn_fill_block_striped_mask.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int64, C.c_int64, C.c_int32, _P(burst_mask_t)]
_lib.burst_attn_visible_pairs.restype = C.c_int64
_lib.burst_attn_visible_pairs.argtypes = [_P(burst_mask_t)]
_lib.burst_attn_tile_class.restype = C.c_int
_lib.burst_attn_tile_class.argtypes = [_P(burst_mask_t)] + [C.c_int64] * 4 + [C.c_int32]
_lib.burst_attn_visible_tile_runs.restype = C.c_int
_lib.burst_attn_visible_tile_runs.argtypes = [_P(burst_mask_t), C.c_int32, C.c_int32, C.c_int64, C.c_int64, _P(C.c_int32 * 4)]
_lib.burst_attn_visible_rows.restype = C.c_int
_lib.burst_attn_visible_rows.argtypes = [_P(burst_mask_t), C.c_int32, C.c_int64, _P(C.c_int32 * 2)]
_lib.burst_attn_set_chunk_rows.restype = C.c_int
_lib.burst_attn_set_chunk_rows.argtypes = [C.c_int32]
_lib.burst_attn_launch_plan.restype = C.c_int
_lib.burst_attn_launch_plan.argtypes = [C.c_int32, C.c_int32, _P(burst_shape_t), _P(burst_mask_t), C.c_int32, _P(C.c_int32)]
_lib.burst_attn_chunk_plan.restype = C.c_int
_lib.burst_attn_chunk_plan.argtypes = [_P(burst_mask_t), C.c_int32, C.c_int32, _P(C.c_int64)]
_lib.burst_attn_mfma_probe.restype = C.c_int
_lib.burst_attn_mfma_probe.argtypes = [C.c_int32, C.c_int32, C.c_void_p, _P(C.c_int64), C.c_void_p]


class burst_lm_head_shape_t(C.Structure):
    _fields_ = [("n_tokens", C.c_int64), ("d_model", C.c_int64), ("vocab", C.c_int64), ("tile_tokens", C.c_int64),
                ("grad_scale", C.c_float), ("_pad", C.c_int32)]


_lib.burst_lm_head_tile_plan.restype = C.c_int
_lib.burst_lm_head_tile_plan.argtypes = [_P(burst_lm_head_shape_t), _P(C.c_int32)]
_lib.burst_lm_head_workspace_bytes.restype = C.c_int64
_lib.burst_lm_head_workspace_bytes.argtypes = [_P(burst_lm_head_shape_t)]
_lib.burst_lm_head_loss.restype = C.c_int
_lib.burst_lm_head_loss.argtypes = [_P(burst_lm_head_shape_t), C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p,
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, C.c_void_p, C.c_int64,
                                    C.c_int32, C.c_void_p, C.c_int64, C.c_void_p]
_lib.burst_lm_head_static_scratch_bytes.restype = C.c_int64
_lib.burst_lm_head_static_scratch_bytes.argtypes = []
_lib.burst_lm_head_loss_noalloc.restype = C.c_int
_lib.burst_lm_head_loss_noalloc.argtypes = [_P(burst_lm_head_shape_t), C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p,
                                            C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, C.c_void_p, C.c_int64,
                                            C.c_int32, C.c_void_p]


class burst_rope_t(C.Structure):
    _fields_ = [("n_axes", C.c_int32), ("rotary_dim", C.c_int32), ("adjacent", C.c_int32), ("_pad", C.c_int32),
                ("inv_freq", C.c_void_p), ("positions", C.c_void_p), ("stride_axis", C.c_int64), ("stride_b", C.c_int64),
                ("axis_of_pair", C.c_uint8 * 64)]


class burst_cache_t(C.Structure):
    _fields_ = [("k", burst_tensor_t), ("v", burst_tensor_t), ("n_pages", C.c_int64), ("page_rows", C.c_int32),
                ("table_cols", C.c_int32), ("table", C.c_void_p), ("table_stride", C.c_int64), ("rows", C.c_void_p),
                ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]


class burst_tree_t(C.Structure):
    _fields_ = [("seen", C.c_void_p), ("seen_stride", C.c_int64), ("first_row", C.c_void_p), ("first_stride", C.c_int64),
                ("tokens", C.c_void_p), ("sink_rows", C.c_int32), ("elsewhere", C.c_int32)]


class burst_scores_shape_t(C.Structure):
    _fields_ = [("n_tokens", C.c_int64), ("vocab", C.c_int64), ("n_top", C.c_int32), ("scale", C.c_float)]


_lib.burst_attn_rope.restype = C.c_int
# (tensors of these calls go in as the bytes of their description)
_lib.burst_attn_rope.argtypes = [_P(burst_shape_t), _P(burst_rope_t)] + [C.c_char_p] * 4 + [C.c_int32, C.c_void_p]
_lib.burst_attn_cache_append.restype = C.c_int
_lib.burst_attn_cache_append.argtypes = [_P(burst_shape_t), _P(burst_cache_t), C.c_char_p, C.c_char_p, C.c_void_p,
                                         _P(burst_rope_t), C.c_char_p, C.c_char_p, C.c_void_p]
_lib.burst_attn_decode_workspace_bytes.restype = C.c_int64
_lib.burst_attn_decode_workspace_bytes.argtypes = [_P(burst_shape_t)]
_lib.burst_attn_decode_plan.restype = C.c_int
_lib.burst_attn_decode_plan.argtypes = [_P(burst_shape_t), _P(burst_cache_t), _P(C.c_int32)]
_lib.burst_attn_decode.restype = C.c_int
_lib.burst_attn_decode.argtypes = [_P(burst_shape_t), _P(burst_cache_t), C.c_char_p, C.c_void_p, C.c_char_p,
                                   C.c_char_p, C.c_void_p, C.c_int64, C.c_void_p]
_lib.burst_attn_tree_workspace_bytes.restype = C.c_int64
_lib.burst_attn_tree_workspace_bytes.argtypes = [_P(burst_shape_t)]
_lib.burst_attn_tree_plan.restype = C.c_int
_lib.burst_attn_tree_plan.argtypes = [_P(burst_shape_t), _P(C.c_int32)]
_lib.burst_attn_tree.restype = C.c_int
_lib.burst_attn_tree.argtypes = [_P(burst_shape_t), _P(burst_cache_t), _P(burst_tree_t), C.c_char_p, C.c_char_p, C.c_char_p, C.c_void_p,
                                 C.c_int64, C.c_void_p]
_lib.burst_attn_cache_copy_pages.restype = C.c_int
_lib.burst_attn_cache_copy_pages.argtypes = [_P(burst_shape_t), C.c_int32, _P(burst_cache_t), C.c_void_p, C.c_int64, C.c_void_p]
_lib.burst_attn_cache_keep_rows.restype = C.c_int
_lib.burst_attn_cache_keep_rows.argtypes = [_P(burst_shape_t), C.c_int32, _P(burst_cache_t), C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                            C.c_void_p]
_lib.burst_lm_head_scores_workspace_bytes.restype = C.c_int64
_lib.burst_lm_head_scores_workspace_bytes.argtypes = [_P(burst_scores_shape_t)]
_lib.burst_lm_head_scores_plan.restype = C.c_int
_lib.burst_lm_head_scores_plan.argtypes = [_P(burst_scores_shape_t), _P(C.c_int32)]
_lib.burst_lm_head_scores_bwd_plan.restype = C.c_int
_lib.burst_lm_head_scores_bwd_plan.argtypes = [_P(burst_scores_shape_t), _P(C.c_int64)]
_lib.burst_lm_head_scores.restype = C.c_int
_lib.burst_lm_head_scores.argtypes = [_P(burst_scores_shape_t), C.c_void_p, C.c_int32, C.c_int64] + [C.c_void_p] * 7 + [C.c_int64, C.c_void_p]
_lib.burst_lm_head_scores_bwd.restype = C.c_int
_lib.burst_lm_head_scores_bwd.argtypes = [_P(burst_scores_shape_t), C.c_void_p, C.c_int32, C.c_int64] + [C.c_void_p] * 9 + [C.c_int32, C.c_int64,
                                                                                                                      C.c_void_p]
_lib.burst_attn_status_string.restype = C.c_char_p
_lib.burst_attn_status_string.argtypes = [C.c_int]
_lib.burst_attn_last_hip_error.restype = C.c_int
_lib.burst_attn_version.restype = C.c_char_p

EXPORTS = ["burst_attn_step_fwd", "burst_attn_steps_fwd", "burst_attn_steps_bwd", "burst_attn_fill_ring_masks",
           "burst_attn_lse_merge", "burst_attn_preprocess_bwd", "burst_attn_step_bwd",
           "burst_attn_fill_zigzag_mask", "burst_attn_fill_contiguous_mask", "burst_attn_fill_striped_mask",
           "burst_attn_fill_block_striped_mask",
           "burst_attn_visible_pairs", "burst_attn_tile_class", "burst_attn_visible_tile_runs", "burst_attn_visible_rows", "burst_attn_mfma_probe", "burst_attn_set_chunk_rows", "burst_attn_chunk_plan", "burst_attn_launch_plan", "burst_attn_status_string", "burst_attn_last_hip_error",
           "burst_attn_version", "burst_lm_head_workspace_bytes", "burst_lm_head_loss",
           "burst_lm_head_static_scratch_bytes", "burst_lm_head_tile_plan", "burst_lm_head_loss_noalloc",
           "burst_attn_rope", "burst_attn_cache_append", "burst_attn_decode_workspace_bytes", "burst_attn_decode", "burst_attn_decode_plan",
           "burst_attn_tree_workspace_bytes", "burst_attn_tree", "burst_attn_tree_plan", "burst_attn_cache_copy_pages", "burst_attn_cache_keep_rows",
           "burst_lm_head_scores_workspace_bytes", "burst_lm_head_scores", "burst_lm_head_scores_bwd", "burst_lm_head_scores_plan", "burst_lm_head_scores_bwd_plan"]


class BurstError(RuntimeError):
    def __init__(self, status):
        self.status = status
        msg = _lib.burst_attn_status_string(status).decode()
        if status == BURST_ERR_HIP:
            msg += f" (hip error {_lib.burst_attn_last_hip_error()})"
        super().__init__(f"libburstattn: {msg}")


def _check(status):
    if status != BURST_OK:
        raise BurstError(status)


def shape(batch, q_heads, kv_heads, head_dim, sq, sk, scale):
    return burst_shape_t(batch, q_heads, kv_heads, head_dim, sq, sk, scale)


def tensor(t):
    """Describe a [batch, seq, heads, head_dim] torch tensor (bf16 or fp32, last dim contiguous)."""
    if t is None:
        return None
    return burst_tensor_t(*_described(t))


_DTYPES = {torch.bfloat16: BURST_BF16, torch.float32: BURST_F32}


def _described(t):
    stride = t.stride()
    assert len(stride) == 4 and stride[3] == 1, "expected [batch, seq, heads, head_dim] with contiguous head_dim"
    return t.data_ptr(), _DTYPES[t.dtype], 0, stride[0], stride[1], stride[2]


def rowvec(t):
    """Describe a [batch, heads, seq] fp32 torch tensor (seq contiguous)."""
    if t is None:
        return None
    stride = t.stride()
    assert len(stride) == 3 and stride[2] == 1 and t.dtype == torch.float32
    return burst_rowvec_t(t.data_ptr(), stride[0], stride[1])


def _ref(x):
    return None if x is None else C.byref(x)


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    return C.c_void_p(stream)


def burst_attn_fill_zigzag_mask(dev_i, shard_j, G, N, causal=True):
    m = burst_mask_t()
    _check(_lib.burst_attn_fill_zigzag_mask(dev_i, shard_j, G, N, int(causal), C.byref(m)))
    return m


def burst_attn_fill_contiguous_mask(dev_i, shard_j, G, N, causal=True):
    m = burst_mask_t()
    _check(_lib.burst_attn_fill_contiguous_mask(dev_i, shard_j, G, N, int(causal), C.byref(m)))
    return m


def burst_attn_fill_striped_mask(dev_i, shard_j, G, N, causal=True):
    m = burst_mask_t()
    _check(_lib.burst_attn_fill_striped_mask(dev_i, shard_j, G, N, int(causal), C.byref(m)))
    return m


def burst_attn_fill_block_striped_mask(dev_i, shard_j, G, N, N_blk, causal=True):
    m = burst_mask_t()
    _check(_lib.burst_attn_fill_block_striped_mask(dev_i, shard_j, G, N, N_blk, int(causal), C.byref(m)))
    return m


_PARTITIONS = {"full": 0, "causal": 1, "zigzag": 2, "striped": 3, "block_striped": 4}


def burst_attn_fill_ring_masks(partition, dev_i, G, N, N_blk=0, window=0):
    """Masks of device dev_i's ring in ring order (its own shard first, then (dev_i - t) mod G): an array of G burst_mask_t."""
    if partition not in _PARTITIONS:
        raise ValueError(partition)
    masks = (burst_mask_t * G)()
    _check(_lib.burst_attn_fill_ring_masks(_PARTITIONS[partition], dev_i, G, N, N_blk, window, masks))
    return masks


def set_block_mask(mask, block_mask, q_block_rows, k_block_rows):
    """Attach a block-wise sparse mask (2-D uint8 device tensor, unit stride along its rows) to a
    burst_mask_t; the tensor must outlive the steps that use the mask."""
    if block_mask.dim() != 2 or block_mask.element_size() != 1 or block_mask.stride(1) != 1 or not block_mask.is_cuda:
        raise ValueError("block_mask: 2-D one-byte device tensor with unit row stride expected")
    mask.block_mask = block_mask.data_ptr()
    mask.q_block_rows, mask.k_block_rows, mask.block_pitch = q_block_rows, k_block_rows, block_mask.stride(0)
    return mask


def burst_attn_visible_pairs(mask):
    return _lib.burst_attn_visible_pairs(C.byref(mask))


def burst_attn_tile_class(mask, q0, q1, k0, k1, method=0):
    st = _lib.burst_attn_tile_class(C.byref(mask), q0, q1, k0, k1, method)
    if st < 0:
        raise BurstError(st)
    return st


def burst_attn_visible_tile_runs(mask, query_axis, tile_rows, r0, r1):
    """Runs of tiles as [(start, length), (start, length)]."""
    out = (C.c_int32 * 4)()
    _check(_lib.burst_attn_visible_tile_runs(C.byref(mask), int(query_axis), tile_rows, r0, r1, C.byref(out)))
    return [(out[0], out[1]), (out[2], out[3])]


def burst_attn_version():
    return _lib.burst_attn_version().decode()


def burst_attn_status_string(status):
    return _lib.burst_attn_status_string(status).decode()


def burst_attn_step_fwd(shp, mask, q, k, v, o_part=None, lse_part=None, o_acc=None, lse_acc=None, stream=None):
    _check(_lib.burst_attn_step_fwd(C.byref(shp), _ref(mask), _ref(tensor(q)), _ref(tensor(k)), _ref(tensor(v)),
                                    _ref(tensor(o_part)), _ref(rowvec(lse_part)), _ref(tensor(o_acc)),
                                    _ref(rowvec(lse_acc)), _stream(stream)))


def burst_attn_lse_merge(shp, o_acc, lse_acc, o_part, lse_part, o_out_cast=None, stream=None):
    _check(_lib.burst_attn_lse_merge(C.byref(shp), _ref(tensor(o_acc)), _ref(rowvec(lse_acc)),
                                     _ref(tensor(o_part)), _ref(rowvec(lse_part)), _ref(tensor(o_out_cast)),
                                     _stream(stream)))


def burst_attn_preprocess_bwd(shp, o, d_o, d_out, stream=None):
    _check(_lib.burst_attn_preprocess_bwd(C.byref(shp), _ref(tensor(o)), _ref(tensor(d_o)), _ref(rowvec(d_out)),
                                          _stream(stream)))


def burst_attn_step_bwd(shp, mask, q, k, v, d_o, lse, d, dq=None, dk=None, dv=None, accumulate_flags=0,
                        stream=None):
    _check(_lib.burst_attn_step_bwd(C.byref(shp), _ref(mask), _ref(tensor(q)), _ref(tensor(k)), _ref(tensor(v)),
                                    _ref(tensor(d_o)), _ref(rowvec(lse)), _ref(rowvec(d)), _ref(tensor(dq)),
                                    _ref(tensor(dk)), _ref(tensor(dv)), accumulate_flags, _stream(stream)))


def _tensor_array(tensors):
    """The bytes of an array of burst_tensor_t."""
    if tensors is None:
        return None
    values = []
    for t in tensors:
        values.extend(_described(t))
    return struct.pack("=" + "Qiiqqq" * len(tensors), *values)


def _mask_array(masks):
    return masks if isinstance(masks, C.Array) else (burst_mask_t * len(masks))(*masks)


def burst_attn_steps_fwd(shapes, masks, q, k, v, o_acc, lse_acc, stream=None):
    """Consecutive steps of one query chunk: shapes, masks, k and v have an entry for each step."""
    n = len(shapes)
    assert len(masks) == n and len(k) == n and len(v) == n
    for i in range(0, n, BURST_MAX_STEPS):
        part = slice(i, i + BURST_MAX_STEPS)
        _check(_lib.burst_attn_steps_fwd(len(shapes[part]), b"".join(shapes[part]), _mask_array(masks if n <= BURST_MAX_STEPS else masks[part]),
                                         _ref(tensor(q)), _tensor_array(k[part]), _tensor_array(v[part]), _ref(tensor(o_acc)),
                                         _ref(rowvec(lse_acc)), _stream(stream)))


def burst_attn_steps_bwd(shapes, masks, q, k, v, d_o, lse, d, dq, dk, dv, accumulate_flags=0, stream=None):
    """Consecutive steps of one query chunk: shapes, masks, k, v, dk and dv have an entry for each step."""
    n = len(shapes)
    assert len(masks) == n and len(k) == n and len(v) == n and all(t is None or len(t) == n for t in (dk, dv))
    for i in range(0, n, BURST_MAX_STEPS):
        part = slice(i, i + BURST_MAX_STEPS)
        _check(_lib.burst_attn_steps_bwd(len(shapes[part]), b"".join(shapes[part]), _mask_array(masks if n <= BURST_MAX_STEPS else masks[part]),
                                         _ref(tensor(q)), _tensor_array(k[part]), _tensor_array(v[part]), _ref(tensor(d_o)),
                                         _ref(rowvec(lse)), _ref(rowvec(d)), _ref(tensor(dq)),
                                         _tensor_array(dk and dk[part]), _tensor_array(dv and dv[part]), accumulate_flags,
                                         _stream(stream)))
        accumulate_flags |= BURST_ACC_DQ


def lm_head_shape(n_tokens, d_model, vocab, tile_tokens, grad_scale=1.0):
    return burst_lm_head_shape_t(n_tokens, d_model, vocab, tile_tokens, grad_scale, 0)


def burst_lm_head_workspace_bytes(shp):
    n = _lib.burst_lm_head_workspace_bytes(C.byref(shp))
    if n < 0:
        raise BurstError(BURST_ERR_INVALID_ARG)
    return n


def burst_lm_head_loss(shp, h_last, w_head, y, loss, workspace, lse=None, d_h=None, d_w=None, accumulate_dw=False,
                       stream=None):
    """h_last [N, d] bf16, w_head [v, d] bf16, y [N] int64, loss / lse [N] fp32, d_h [N, d] fp32 or bf16,
    d_w [v, d] fp32, workspace: one-byte tensor of burst_lm_head_workspace_bytes(shp) bytes.  Rows may be
    strided; the last dimension is contiguous."""
    for t in (h_last, w_head, d_h, d_w):
        assert t is None or (t.dim() == 2 and t.stride(1) == 1), "expected 2-D tensors with a contiguous last dim"
    assert h_last.dtype == torch.bfloat16 and w_head.dtype == torch.bfloat16 and y.dtype == torch.int64
    assert y.is_contiguous() and loss.is_contiguous() and loss.dtype == torch.float32
    assert lse is None or (lse.is_contiguous() and lse.dtype == torch.float32)
    assert d_w is None or d_w.dtype == torch.float32
    ptr = lambda t: None if t is None else C.c_void_p(t.data_ptr())
    dh_dtype = BURST_F32 if d_h is None else {torch.bfloat16: BURST_BF16, torch.float32: BURST_F32}[d_h.dtype]
    _check(_lib.burst_lm_head_loss(C.byref(shp), ptr(h_last), h_last.stride(0), ptr(w_head), w_head.stride(0), ptr(y),
                                   ptr(loss), ptr(lse), ptr(d_h), dh_dtype, 0 if d_h is None else d_h.stride(0),
                                   ptr(d_w), 0 if d_w is None else d_w.stride(0), int(accumulate_dw),
                                   ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))


def burst_lm_head_static_scratch_bytes():
    """The workspace that a shape may need for burst_lm_head_loss_noalloc (the array itself is larger)."""
    return _lib.burst_lm_head_static_scratch_bytes()


def burst_lm_head_loss_noalloc(shp, h_last, w_head, y, loss, lse=None, d_h=None, d_w=None, accumulate_dw=False,
                               stream=None):
    """burst_lm_head_loss on the library's built-in scratch array (no workspace argument, no allocation)."""
    for t in (h_last, w_head, d_h, d_w):
        assert t is None or (t.dim() == 2 and t.stride(1) == 1), "expected 2-D tensors with a contiguous last dim"
    assert h_last.dtype == torch.bfloat16 and w_head.dtype == torch.bfloat16 and y.dtype == torch.int64
    assert y.is_contiguous() and loss.is_contiguous() and loss.dtype == torch.float32
    assert lse is None or (lse.is_contiguous() and lse.dtype == torch.float32)
    assert d_w is None or d_w.dtype == torch.float32
    ptr = lambda t: None if t is None else C.c_void_p(t.data_ptr())
    dh_dtype = BURST_F32 if d_h is None else {torch.bfloat16: BURST_BF16, torch.float32: BURST_F32}[d_h.dtype]
    _check(_lib.burst_lm_head_loss_noalloc(C.byref(shp), ptr(h_last), h_last.stride(0), ptr(w_head), w_head.stride(0),
                                           ptr(y), ptr(loss), ptr(lse), ptr(d_h), dh_dtype,
                                           0 if d_h is None else d_h.stride(0), ptr(d_w),
                                           0 if d_w is None else d_w.stride(0), int(accumulate_dw), _stream(stream)))


def burst_attn_visible_rows(mask, query_axis, row):
    """(lo, hi): rows of the query axis that see key row `row`, or of the key axis that query row `row` sees."""
    out = (C.c_int32 * 2)()
    _check(_lib.burst_attn_visible_rows(C.byref(mask), int(query_axis), int(row), C.byref(out)))
    return out[0], out[1]


def burst_attn_set_chunk_rows(rows):
    """Rows of the streamed axis per launch of a step kernel (diagnostics); returns the value in force."""
    return _lib.burst_attn_set_chunk_rows(int(rows))


def burst_attn_chunk_plan(mask, query_axis, max_ranges=4096):
    """Ranges the step launchers cut an axis into: list of dicts (r0, r1, nseg, seg_len, pos0, period, blk_offset)."""
    out = (C.c_int64 * (7 * max_ranges))()
    n = _lib.burst_attn_chunk_plan(C.byref(mask), int(query_axis), max_ranges, out)
    if n < 0:
        _check(n)
    keys = ("r0", "r1", "nseg", "seg_len", "pos0", "period", "blk_offset")
    return [dict(zip(keys, out[7 * i:7 * i + 7])) for i in range(min(n, max_ranges))]


def burst_attn_launch_plan(call, shapes, masks, max_launches=4096):
    """Kernels (BURST_KERNEL_ bits) of the launches of a call; call: "fwd", "fwd_part", "bwd", "dq" or "dkdv"."""
    out = (C.c_int32 * max_launches)()
    n = _lib.burst_attn_launch_plan(("fwd", "fwd_part", "bwd", "dq", "dkdv").index(call), len(shapes), (burst_shape_t * len(shapes))(*shapes),
                                    (burst_mask_t * len(masks))(*masks), max_launches, out)
    if n < 0:
        _check(n)
    return list(out[:min(n, max_launches)])


def burst_lm_head_tile_plan(shp):
    """(edge of an output tile, parts of its contraction) of the logits, dH and dW of the first sequence tile."""
    out = (C.c_int32 * 6)()
    _check(_lib.burst_lm_head_tile_plan(C.byref(shp), out))
    return [tuple(out[2 * i:2 * i + 2]) for i in range(3)]


def _current(stream):
    """The stream to use (the current one, or a given one of the current device) and the number of its device."""
    device = torch.cuda.current_device()
    # (the handle alone: torch.cuda.current_stream() makes an object of it, 2.8 us of the 9 that a call took)
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream, device


def _check_device(device, *tensors):
    """Kernels run on the current device: tensors that are elsewhere are refused."""
    for t in tensors:
        if t is not None and t.get_device() != device:      # (-1: not on a GPU)
            raise ValueError(f"tensor on {t.device}, the current device is cuda:{device}")


_pack_tensor, _pack_rowvec = struct.Struct("=Qiiqqq").pack, struct.Struct("=Qqq").pack


def _packed(t, device, sizes):
    """The bytes of the burst_tensor_t of a tensor of these sizes on this device, or None."""
    if t is None:
        return None
    stride = t.stride()
    if t.shape != sizes or stride[3] != 1:
        raise ValueError(f"tensor of {sizes} with a contiguous last dimension expected, not {tuple(t.shape)}, strides {stride}")
    if t.get_device() != device:
        _check_device(device, t)
    return _pack_tensor(t.data_ptr(), _DTYPES[t.dtype], 0, stride[0], stride[1], stride[2])


def _int32(t, dims):
    if t.dtype != torch.int32 or t.dim() != dims or (t.numel() > 0 and t.size(-1) > 1 and t.stride(-1) != 1):
        raise ValueError(f"int32 tensor of {dims} dimensions with a contiguous last one expected")
    return t.data_ptr()


def rope(positions, inv_freq, rotary_dim=None, adjacent=False, axis_of_pair=None):
    """A rotation: positions [axes, batch, rows] int32, inv_freq [rotary_dim / 2] fp32, the axis of each pair (default: the first).  A
    plan that a program keeps: it holds the two tensors, whose contents are read when a call that uses it runs."""
    device = torch.cuda.current_device()
    _check_device(device, positions, inv_freq)
    pairs = inv_freq.numel()
    if inv_freq.dtype != torch.float32 or not inv_freq.is_contiguous() or (rotary_dim is not None and rotary_dim != 2 * pairs):
        raise ValueError("inv_freq: rotary_dim / 2 contiguous fp32 numbers expected")
    axes = [0] * pairs if axis_of_pair is None else [int(a) for a in axis_of_pair]
    if len(axes) != pairs or not all(0 <= a < positions.size(0) for a in axes):
        raise ValueError("axis_of_pair: an axis of positions for each pair expected")
    if pairs > 64:
        raise ValueError("at most 64 pairs")
    r = burst_rope_t(positions.size(0), 2 * pairs, int(adjacent), 0, inv_freq.data_ptr(), _int32(positions, 3),
                     positions.stride(0), positions.stride(1), (C.c_uint8 * 64)(*axes))
    r._tensors, r._rows, r._device = (positions, inv_freq), tuple(positions.shape[1:]), device
    return r


def _elsewhere(handle, device):
    """A rotation or a cache is used where its tensors are."""
    return ValueError(f"made on cuda:{handle._device}, the current device is cuda:{device}")


def _check_positions(r, batch, sq, device):
    if r is None:
        return
    if r._device != device:
        raise _elsewhere(r, device)
    if r._rows != (batch, sq):
        raise ValueError(f"positions of {batch} sequences of {sq} rows expected, not {r._rows}")


def burst_attn_rope(shp, rope, q, q_out, k=None, k_out=None, inverse=False, stream=None):
    """q, q_out [batch, sq, q_heads, head_dim], k, k_out [batch, sq, kv_heads, head_dim], bf16 or fp32; q_out may be q (in place)."""
    stream, device = _current(stream)
    batch, sq, d = shp.batch, shp.sq, shp.head_dim
    q_sizes, k_sizes = (batch, sq, shp.q_heads, d), (batch, sq, shp.kv_heads, d)
    _check_positions(rope, batch, sq, device)
    _check(_lib.burst_attn_rope(shp, rope, _packed(q, device, q_sizes), _packed(q_out, device, q_sizes), _packed(k, device, k_sizes),
                                _packed(k_out, device, k_sizes), int(inverse), stream))


def paged_cache(k, v, table, rows, k_scale=None, v_scale=None):
    """A paged cache: k and v [pages, page_rows, kv_heads, head_dim] (bf16 or float8_e4m3fn, in any order of memory), table int32
    [batch, pages of a sequence], rows int32 [batch], scales fp32 [kv_heads].  A handle that a program keeps; it holds the tensors."""
    device = torch.cuda.current_device()
    _check_device(device, k, v, table, rows, k_scale, v_scale)
    if k.shape != v.shape or k.dim() != 4 or table.dim() != 2 or rows.dim() != 1 or table.size(0) != rows.size(0):
        raise ValueError("k and v [pages, page_rows, kv_heads, head_dim], table [batch, pages], rows [batch] expected")
    if rows.numel() > 1 and rows.stride(0) != 1:
        raise ValueError("rows: contiguous numbers expected")
    for s in (k_scale, v_scale):
        if s is not None and (s.dtype != torch.float32 or not s.is_contiguous() or s.numel() != k.size(2)):
            raise ValueError("scales: kv_heads contiguous fp32 numbers expected")
    c = burst_cache_t(_cache_tensor(k), _cache_tensor(v), k.size(0), k.size(1), table.size(1), _int32(table, 2),
                      table.stride(0) if table.size(0) > 1 else 0,
                      _int32(rows, 1), None if k_scale is None else k_scale.data_ptr(), None if v_scale is None else v_scale.data_ptr())
    c._tensors, c._sizes, c._device = (k, v, table, rows, k_scale, v_scale), (rows.size(0), k.size(2), k.size(3)), device
    return c


def _cache_tensor(t):
    if t.stride(3) != 1:
        raise ValueError("head_dim must be contiguous")
    return burst_tensor_t(t.data_ptr(), {torch.bfloat16: BURST_BF16, torch.float8_e4m3fn: BURST_F8E4M3}[t.dtype], 0, t.stride(0),
                          t.stride(1), t.stride(2))


def _check_cache(cache, batch, kv_heads, d, device):
    if cache._device != device:
        raise _elsewhere(cache, device)
    if cache._sizes != (batch, kv_heads, d):
        raise ValueError("the cache has another batch, kv_heads or head_dim than the shape")


def _numbers(t, device, batch):
    """The address of an int32 number for each sequence, or None."""
    if t is None:
        return None
    if t.get_device() != device:
        _check_device(device, t)
    if t.dtype != torch.int32 or t.shape != (batch,) or (batch > 1 and t.stride(0) != 1):
        raise ValueError(f"int32 tensor of {(batch,)} contiguous numbers expected, not {t.dtype} {tuple(t.shape)}, strides {t.stride()}")
    return t.data_ptr()


def burst_attn_cache_append(shp, cache, k, v, new_rows=None, rope=None, q=None, q_out=None, stream=None):
    """k, v [batch, sq, kv_heads, head_dim] bf16: sequence b's first new_rows[b] rows (all) become its rows rows[b] - new_rows[b] ..
    rows[b] - 1.  With a rotation the keys are turned, and q [batch, sq, q_heads, head_dim] into q_out."""
    stream, device = _current(stream)
    batch, sq, kv_heads, d = shp.batch, shp.sq, shp.kv_heads, shp.head_dim
    q_sizes, k_sizes = (batch, sq, shp.q_heads, d), (batch, sq, kv_heads, d)
    _check_cache(cache, batch, kv_heads, d, device)
    _check_positions(rope, batch, sq, device)
    _check(_lib.burst_attn_cache_append(shp, cache, _packed(k, device, k_sizes), _packed(v, device, k_sizes),
                                        _numbers(new_rows, device, batch), rope, _packed(q, device, q_sizes),
                                        _packed(q_out, device, q_sizes), stream))


def burst_attn_decode_workspace_bytes(shp):
    n = _lib.burst_attn_decode_workspace_bytes(C.byref(shp))
    if n < 0:
        raise BurstError(BURST_ERR_INVALID_ARG)
    return n


def burst_attn_decode(shp, cache, q, o, lse=None, workspace=None, first_row=None, stream=None):
    """q [batch, 1, q_heads, head_dim] bf16 over the cache's rows from first_row[b] on: o (bf16 or fp32), lse [batch, q_heads, 1].
    shp.sk bounds the rows of a sequence; workspace: a one-byte tensor of burst_attn_decode_workspace_bytes(shp) bytes."""
    stream, device = _current(stream)
    batch, q_heads, kv_heads, d = shp.batch, shp.q_heads, shp.kv_heads, shp.head_dim
    _check_cache(cache, batch, kv_heads, d, device)
    sizes, ws, n = (batch, 1, q_heads, d), None, 0
    if lse is not None:
        stride = lse.stride()
        if lse.shape != (batch, q_heads, 1) or lse.dtype != torch.float32:
            raise ValueError(f"lse: fp32 tensor of {(batch, q_heads, 1)} expected")
        if lse.get_device() != device:
            _check_device(device, lse)
        lse = _pack_rowvec(lse.data_ptr(), stride[0], stride[1])
    if workspace is not None:
        if workspace.get_device() != device:
            _check_device(device, workspace)
        ws, n = workspace.data_ptr(), workspace.nbytes
    _check(_lib.burst_attn_decode(shp, cache, _packed(q, device, sizes), _numbers(first_row, device, batch), _packed(o, device, sizes),
                                  lse, ws, n, stream))


def burst_attn_decode_plan(shp, cache):
    """(shares, key heads that a work-group takes together, whether nothing is dealt) of a burst_attn_decode (diagnostics)."""
    out = (C.c_int32 * 3)()
    _check(_lib.burst_attn_decode_plan(shp, cache, out))
    return out[0], out[1], bool(out[2])


def tree(seen=None, first_row=None, tokens=None, sink_rows=0, elsewhere=False):
    """What new tokens see: seen int64 [batch, sq] (the bits of a word for each token; None: a chain), first_row int32 [batch, sq] (of the older rows),
    tokens int32 [batch] (how many a sequence brings; None: sq), the first sink_rows rows always, elsewhere: their own rows are in another cache.
    A plan that a program keeps; it holds the tensors, whose contents are read when a call that uses it runs."""
    device = torch.cuda.current_device()
    _check_device(device, seen, first_row, tokens)
    if not 0 <= sink_rows < 1 << 31:
        raise ValueError(f"sink_rows: a number of 0 to 2^31 - 1 rows expected, not {sink_rows}")
    t = burst_tree_t(None, 0, None, 0, None, sink_rows, int(elsewhere))
    sizes = [None, None]                # batch, sq: of the tensors that there are
    for name, x, dtype in (("seen", seen, torch.int64), ("first_row", first_row, torch.int32), ("tokens", tokens, torch.int32)):
        if x is None:
            continue
        dims = 1 if name == "tokens" else 2
        if x.dtype != dtype or x.dim() != dims or (x.size(-1) > 1 and x.stride(-1) != 1):
            raise ValueError(f"{name}: {dtype} tensor of {dims} dimensions with a contiguous last one expected")
        for i, n in enumerate(x.shape):
            if sizes[i] not in (None, n):
                raise ValueError("seen and first_row [batch, sq], tokens [batch] expected")
            sizes[i] = n
        setattr(t, name, x.data_ptr())
        if dims == 2:
            setattr(t, "seen_stride" if name == "seen" else "first_stride", x.stride(0) if x.size(0) > 1 else 0)
    t._tensors, t._sizes, t._device = (seen, first_row, tokens), tuple(sizes), device
    return t


def burst_attn_tree_workspace_bytes(shp):
    n = _lib.burst_attn_tree_workspace_bytes(C.byref(shp))
    if n < 0:
        raise BurstError(BURST_ERR_INVALID_ARG)
    return n


def burst_attn_tree(shp, cache, tree, q, o, lse=None, workspace=None, stream=None):
    """q [batch, sq, q_heads, head_dim] bf16, new tokens of every sequence, over the cache's rows that the tree says: o (bf16 or fp32), lse [batch,
    q_heads, sq].  shp.sk bounds the rows of a sequence; workspace: a one-byte tensor of burst_attn_tree_workspace_bytes(shp) bytes."""
    stream, device = _current(stream)
    batch, sq, q_heads, kv_heads, d = shp.batch, shp.sq, shp.q_heads, shp.kv_heads, shp.head_dim
    _check_cache(cache, batch, kv_heads, d, device)
    if tree._device != device:
        raise _elsewhere(tree, device)
    if tree._sizes[0] not in (None, batch) or tree._sizes[1] not in (None, sq):
        raise ValueError(f"the tree is of {tree._sizes}, not of {(batch, sq)} sequences and tokens")
    sizes, ws, n = (batch, sq, q_heads, d), None, 0
    if lse is not None:
        stride = lse.stride()
        if lse.shape != (batch, q_heads, sq) or lse.dtype != torch.float32 or (sq > 1 and stride[2] != 1):
            raise ValueError(f"lse: fp32 tensor of {(batch, q_heads, sq)} with a contiguous last dimension expected")
        if lse.get_device() != device:
            _check_device(device, lse)
        lse = _pack_rowvec(lse.data_ptr(), stride[0], stride[1])
    if workspace is not None:
        if workspace.get_device() != device:
            _check_device(device, workspace)
        ws, n = workspace.data_ptr(), workspace.nbytes
    _check(_lib.burst_attn_tree(shp, cache, tree, _packed(q, device, sizes), _packed(o, device, sizes), lse, ws, n, stream))


def burst_attn_tree_plan(shp):
    """(shares, columns of a work-group, whether nothing is dealt) of a burst_attn_tree (diagnostics)."""
    out = (C.c_int32 * 3)()
    _check(_lib.burst_attn_tree_plan(shp, out))
    return out[0], out[1], bool(out[2])


def cache_layers(caches):
    """Caches of a model's layers (paged_cache), for calls that move pages or rows in all of them.  A handle that a program keeps; it holds them."""
    caches = list(caches)
    if not caches or any(c._device != caches[0]._device or c._sizes != caches[0]._sizes for c in caches):
        raise ValueError("caches of one device, batch, kv_heads and head_dim expected")
    layers = (burst_cache_t * len(caches))(*caches)
    layers._caches, layers._device = caches, caches[0]._device
    batch, kv_heads, d = caches[0]._sizes
    # (for 0 .. 64 new rows, made once: a structure takes 0.8 us of a call)
    layers._shapes = [burst_shape_t(batch, kv_heads, kv_heads, d, sq, 0, 1.0) for sq in range(BURST_TREE_MAX_TOKENS + 2)]
    layers._per_sequence = (batch,)
    return layers


def burst_attn_cache_copy_pages(layers, moves, stream=None):
    """moves int32 [n, 3]: from, to, rows: the first rows of a page to another page, in all layers."""
    stream, device = _current(stream)
    if layers._device != device:
        raise _elsewhere(layers, device)
    if moves.get_device() != device:
        _check_device(device, moves)
    if moves.dtype != torch.int32 or moves.dim() != 2 or moves.size(1) != 3 or not moves.is_contiguous():
        raise ValueError("moves: contiguous int32 tensor of [n, 3] expected")
    _check(_lib.burst_attn_cache_copy_pages(layers._shapes[0], len(layers), layers, moves.data_ptr(), moves.size(0), stream))


def burst_attn_cache_keep_rows(layers, from_rows, kept, new_rows=None, stream=None):
    """from_rows int32 [batch, sq]: of a sequence's last new_rows[b] rows (sq) row from_rows[b][i] becomes row i, for i < kept[b], in all layers."""
    stream, device = _current(stream)
    if layers._device != device:
        raise _elsewhere(layers, device)
    if from_rows.get_device() != device:
        _check_device(device, from_rows)
    sizes, stride, n = from_rows.shape, from_rows.stride(), layers._per_sequence
    if from_rows.dtype is not torch.int32 or len(sizes) != 2 or sizes[0] != n[0] or (sizes[1] > 1 and stride[1] != 1):
        raise ValueError(f"from_rows: int32 tensor of [{n[0]}, sq] with a contiguous last dimension expected, not {from_rows.dtype} {tuple(sizes)}, strides {stride}")
    shp = layers._shapes[min(sizes[1], BURST_TREE_MAX_TOKENS + 1)]   # (more are refused)
    _check(_lib.burst_attn_cache_keep_rows(shp, len(layers), layers, from_rows.data_ptr(), stride[0] if sizes[0] > 1 else 0,
                                           _per_token(new_rows, torch.int32, n, device), _per_token(kept, torch.int32, n, device), stream))


def scores_shape(n_tokens, vocab, n_top=0, scale=1.0):
    return burst_scores_shape_t(n_tokens, vocab, n_top, scale)


def burst_lm_head_scores_workspace_bytes(shp):
    n = _lib.burst_lm_head_scores_workspace_bytes(C.byref(shp))
    if n < 0:
        raise BurstError(BURST_ERR_INVALID_ARG)
    return n


def burst_lm_head_scores_plan(shp):
    """(waves that take a part of a row together, parts of a row) of a burst_lm_head_scores (diagnostics)."""
    out = (C.c_int32 * 2)()
    _check(_lib.burst_lm_head_scores_plan(shp, out))
    return out[0], out[1]


def burst_lm_head_scores_bwd_plan(shp):
    """Tokens that a launch of a burst_lm_head_scores_bwd takes at most (diagnostics)."""
    out = (C.c_int64 * 1)()
    _check(_lib.burst_lm_head_scores_bwd_plan(shp, out))
    return out[0]


def _logits(t, shp, device, name):
    """Address, type and row stride of a matrix of logits or of their gradient."""
    n, v = shp.n_tokens, shp.vocab
    if t.shape != (n, v) or (v > 1 and t.stride(1) != 1):
        raise ValueError(f"{name}: tensor of {(n, v)} with a contiguous last dimension expected, not {tuple(t.shape)}, strides {t.stride()}")
    if t.get_device() != device:
        _check_device(device, t)
    return t.data_ptr(), _DTYPES[t.dtype], t.stride(0) if n > 1 else v


def _per_token(t, dtype, sizes, device):
    """The address of a contiguous tensor of these sizes, or None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != sizes or not t.is_contiguous():
        raise ValueError(f"contiguous {dtype} tensor of {sizes} expected, not {t.dtype} {tuple(t.shape)}, strides {t.stride()}")
    if t.get_device() != device:
        _check_device(device, t)
    return t.data_ptr()


def burst_lm_head_scores(shp, logits, y=None, logp=None, lse=None, entropy=None, top_logp=None, top_ids=None, workspace=None, stream=None):
    """logits [n, vocab] bf16 or fp32 (rows may be strided), y int64 [n]: logp, lse, entropy fp32 [n], top_logp fp32 and top_ids int64 [n, n_top];
    workspace: a one-byte tensor of burst_lm_head_scores_workspace_bytes(shp) bytes."""
    stream, device = _current(stream)
    n, ws, ws_bytes = (shp.n_tokens,), None, 0
    top = (shp.n_tokens, shp.n_top)
    if workspace is not None:
        if workspace.get_device() != device:
            _check_device(device, workspace)
        ws, ws_bytes = workspace.data_ptr(), workspace.nbytes
    f32, i64 = torch.float32, torch.int64
    _check(_lib.burst_lm_head_scores(shp, *_logits(logits, shp, device, "logits"), _per_token(y, i64, n, device), _per_token(logp, f32, n, device),
                                     _per_token(lse, f32, n, device), _per_token(entropy, f32, n, device), _per_token(top_logp, f32, top, device),
                                     _per_token(top_ids, i64, top, device), ws, ws_bytes, stream))


def burst_lm_head_scores_bwd(shp, logits, lse, d_logits, y=None, entropy=None, top_ids=None, g_logp=None, g_lse=None, g_entropy=None, g_top=None,
                             stream=None):
    """The gradient of the logits, d_logits [n, vocab] bf16 or fp32 (logits itself, too), from those of the scores: g_logp, g_lse, g_entropy fp32
    [n], g_top fp32 [n, n_top]."""
    stream, device = _current(stream)
    n, top = (shp.n_tokens,), (shp.n_tokens, shp.n_top)
    f32, i64 = torch.float32, torch.int64
    _check(_lib.burst_lm_head_scores_bwd(shp, *_logits(logits, shp, device, "logits"), _per_token(y, i64, n, device), _per_token(lse, f32, n, device),
                                         _per_token(entropy, f32, n, device), _per_token(top_ids, i64, top, device),
                                         _per_token(g_logp, f32, n, device), _per_token(g_lse, f32, n, device), _per_token(g_entropy, f32, n, device),
                                         _per_token(g_top, f32, top, device), *_logits(d_logits, shp, device, "d_logits"), stream))


def burst_attn_mfma_probe(random_operands, iterations, stream=None):
    """Enqueue the MFMA ceiling probe; returns the flop count of the launch."""
    flops = C.c_int64(0)
    _check(_lib.burst_attn_mfma_probe(int(random_operands), iterations, None, C.byref(flops), _stream(stream)))
    return flops.value


def raw():
    """The ctypes library handle, for tests that exercise the error paths with raw structs."""
    return _lib
