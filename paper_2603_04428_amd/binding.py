"""ctypes binding of libq4kv.so: the same entry points as include/q4kv.h, taking torch tensors.

Argument marshalling only -- pointers, sizes and the current HIP stream are handed to the C ABI;
every step of the path runs in the library's kernels.  There is no fallback: if the shared
library is missing or a call fails, an exception is raised.
"""
import ctypes as C
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libq4kv.so")

EXPORTS = ["q4kv_quantize", "q4kv_dequantize", "q4kv_quantize_fmt", "q4kv_dequantize_fmt", "q4kv_append", "q4kv_batched_attention",
           "q4kv_batched_attention_windows", "q4kv_batched_attention_static", "q4kv_decode_plan",
           "q4kv_batched_attention_planned", "q4kv_attention_workspace_bytes", "q4kv_default_split_tokens", "q4kv_cache_bytes", "q4kv_block_image_bytes", "q4kv_export_blocks", "q4kv_import_blocks", "q4kv_read_probe",
           "q4kv_block_pool_create", "q4kv_block_pool_destroy", "q4kv_block_pool_reserve", "q4kv_block_pool_release",
           "q4kv_block_pool_blocks", "q4kv_block_pool_table_row", "q4kv_block_pool_touch", "q4kv_block_pool_pin",
           "q4kv_block_pool_lru_victim", "q4kv_block_pool_free_blocks", "q4kv_block_pool_owner",
           "q4kv_block_pool_fork", "q4kv_block_pool_truncate", "q4kv_block_pool_compact", "q4kv_block_pool_shares",
           "q4kv_copy_blocks", "q4kv_norm_rope_append", "q4kv_shared_prefix_attention", "q4kv_shared_prefix_workspace_bytes",
           "q4kv_append_slots", "q4kv_resize_tables", "q4kv_beam_reorder", "q4kv_tables_workspace_bytes", "q4kv_beam_select",
           "q4kv_beam_select_workspace_bytes", "q4kv_last_error",
           "q4kv_version"]


class Q4KVError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"libq4kv error {code}: {msg}")
        self.code = code


class Spec(C.Structure):
    """q4kv_spec"""
    _fields_ = [("num_layers", C.c_int32), ("num_q_heads", C.c_int32), ("num_kv_heads", C.c_int32),
                ("k_dim", C.c_int32), ("v_dim", C.c_int32), ("v_aliases_k", C.c_int32),
                ("block_tokens", C.c_int32), ("group_size", C.c_int32), ("param_format", C.c_int32)]


PARAMS_F16, PARAMS_BF16 = 0, 1   # q4kv_param_format: type of the stored scale and bias


class _CPool(C.Structure):
    """q4kv_pool"""
    _fields_ = [("codes", C.c_void_p), ("scale", C.c_void_p), ("bias", C.c_void_p), ("num_blocks", C.c_int32)]


class _CHeadForm(C.Structure):
    """q4kv_head_form"""
    _fields_ = [("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("cos_table", C.c_void_p), ("sin_table", C.c_void_p),
                ("norm_dim", C.c_int32), ("eps", C.c_float), ("rot_begin", C.c_int32), ("rot_dim", C.c_int32),
                ("neighbours", C.c_int32), ("table_len", C.c_int32)]


class _CTables(C.Structure):
    """q4kv_tables"""
    _fields_ = [("block_table", C.c_void_p), ("seq_len", C.c_void_p), ("refs", C.c_void_p), ("refused", C.c_void_p),
                ("num_agents", C.c_int32), ("max_blocks", C.c_int32), ("num_blocks", C.c_int32)]


_lib = None


def lib():
    """Load libq4kv.so (built in-tree by paper_2603_04428_amd/build.py); raise if it is not there."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'` "
                              "(there is no fallback path)")
        l = C.CDLL(LIB_PATH)
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        l.q4kv_quantize.argtypes = [vp, i64, i32, vp, vp, vp, vp]
        l.q4kv_dequantize.argtypes = [vp, vp, vp, i64, i32, vp, vp]
        l.q4kv_quantize_fmt.argtypes = [vp, i64, i32, i32, vp, vp, vp, vp]
        l.q4kv_dequantize_fmt.argtypes = [vp, vp, vp, i64, i32, i32, vp, vp]
        l.q4kv_append.argtypes = [C.POINTER(Spec), C.POINTER(_CPool), C.POINTER(_CPool), vp, vp, vp, i32, vp, i32, i32,
                                  i32, i32, vp]
        l.q4kv_batched_attention.argtypes = [C.POINTER(Spec), C.POINTER(_CPool), C.POINTER(_CPool), vp, vp, vp, i32, vp,
                                             i32, i32, i32, C.c_float, i32, i32, i32, i32, vp, C.c_size_t, vp]
        l.q4kv_batched_attention_windows.argtypes = [C.POINTER(Spec), C.POINTER(_CPool), C.POINTER(_CPool), vp, vp, vp,
                                                     i32, vp, i32, i32, i32, C.c_float, C.POINTER(i32), i32, i32, i32,
                                                     vp, C.c_size_t, vp]
        l.q4kv_batched_attention_static.argtypes = [C.POINTER(Spec), C.POINTER(_CPool), C.POINTER(_CPool), vp, vp, vp, i32,
                                                    vp, i32, i32, i32, C.c_float, i32, i32, i32, i32, vp]
        l.q4kv_decode_plan.argtypes = [C.POINTER(Spec), vp, i32, i32, i32, i32, i32, vp, C.c_size_t, vp]
        l.q4kv_batched_attention_planned.argtypes = [C.POINTER(Spec), C.POINTER(_CPool), C.POINTER(_CPool), vp, vp, vp, i32,
                                                     i32, i32, C.c_float, i32, i32, i32, i32, vp, C.c_size_t, vp]
        l.q4kv_attention_workspace_bytes.restype = C.c_size_t
        l.q4kv_attention_workspace_bytes.argtypes = [C.POINTER(Spec), i32, i32, i32, i32, i32]
        l.q4kv_default_split_tokens.restype = i32
        l.q4kv_default_split_tokens.argtypes = [C.POINTER(Spec), i32, i32, i32, i32]
        l.q4kv_cache_bytes.restype = i64
        l.q4kv_cache_bytes.argtypes = [C.POINTER(Spec), i64]
        l.q4kv_read_probe.argtypes = [vp, C.c_size_t, vp, vp]
        l.q4kv_block_image_bytes.restype = C.c_size_t
        l.q4kv_block_image_bytes.argtypes = [C.POINTER(Spec), i32]
        for f in (l.q4kv_export_blocks, l.q4kv_import_blocks):
            f.argtypes = [C.POINTER(Spec), C.POINTER(_CPool), C.POINTER(_CPool), vp, i32, vp, C.c_size_t, vp]
        l.q4kv_block_pool_create.restype = vp
        l.q4kv_block_pool_create.argtypes = [i32]
        l.q4kv_block_pool_destroy.restype = None
        l.q4kv_block_pool_destroy.argtypes = [vp]
        l.q4kv_block_pool_reserve.argtypes = [vp, i64, i64]
        l.q4kv_block_pool_release.argtypes = [vp, i64]
        l.q4kv_block_pool_blocks.argtypes = [vp, i64, C.POINTER(i32), i32]
        l.q4kv_block_pool_table_row.argtypes = [vp, i64, C.POINTER(i32), i32, i32]
        l.q4kv_block_pool_touch.argtypes = [vp, i64]
        l.q4kv_block_pool_pin.argtypes = [vp, i64, i32]
        l.q4kv_block_pool_lru_victim.restype = i64
        l.q4kv_block_pool_lru_victim.argtypes = [vp]
        l.q4kv_block_pool_free_blocks.argtypes = [vp]
        l.q4kv_block_pool_owner.restype = i64
        l.q4kv_block_pool_owner.argtypes = [vp, i32]
        l.q4kv_block_pool_fork.argtypes = [vp, i64, i64, i64, C.POINTER(i32), C.POINTER(i32)]
        l.q4kv_block_pool_truncate.argtypes = [vp, i64, i64, C.POINTER(i32), C.POINTER(i32)]
        l.q4kv_block_pool_compact.argtypes = [vp, C.POINTER(i32), C.POINTER(i32), i32]
        l.q4kv_block_pool_shares.argtypes = [vp, i32]
        l.q4kv_copy_blocks.argtypes = [C.POINTER(Spec), C.POINTER(_CPool), C.POINTER(_CPool), vp, vp, i32, vp]
        l.q4kv_norm_rope_append.argtypes = [C.POINTER(Spec), C.POINTER(_CPool), C.POINTER(_CPool), C.POINTER(_CHeadForm), vp, vp, vp,
                                            i32, i64, i64, i64, vp, vp, i32, vp, vp, i32, i32, i32, i32, vp]
        l.q4kv_shared_prefix_attention.argtypes = [C.POINTER(Spec), C.POINTER(_CPool), C.POINTER(_CPool), vp, vp, vp, i32, vp, i32, vp, vp,
                                                   i32, i32, C.c_float, i32, i32, vp, C.c_size_t, vp]
        l.q4kv_shared_prefix_workspace_bytes.restype = C.c_size_t
        l.q4kv_shared_prefix_workspace_bytes.argtypes = [C.POINTER(Spec), i32, i32, i32]
        l.q4kv_append_slots.argtypes = [C.POINTER(Spec), C.POINTER(_CPool), C.POINTER(_CPool), vp, vp, i32, i64, i64, vp, i32, i32, i32, vp]
        l.q4kv_resize_tables.argtypes = [C.POINTER(_CTables), vp, i32, vp, vp, vp, vp, C.POINTER(Spec), C.POINTER(_CPool), C.POINTER(_CPool),
                                         vp, C.c_size_t, vp]
        l.q4kv_beam_reorder.argtypes = [C.POINTER(Spec), C.POINTER(_CPool), C.POINTER(_CPool), C.POINTER(_CTables), vp, vp, C.c_size_t, vp]
        l.q4kv_tables_workspace_bytes.restype = C.c_size_t
        l.q4kv_tables_workspace_bytes.argtypes = [i32]
        l.q4kv_beam_select.argtypes = [vp, i32, i64, i32, i32, vp, vp, vp, i32, i32, vp, vp, vp, vp, C.c_size_t, vp]
        l.q4kv_beam_select_workspace_bytes.restype = C.c_size_t
        l.q4kv_beam_select_workspace_bytes.argtypes = [i32, i32, i32, i32]
        l.q4kv_last_error.restype = C.c_char_p
        l.q4kv_version.restype = C.c_int
        _lib = l
    return _lib


def _check(rc):
    if rc != 0:
        raise Q4KVError(rc, lib().q4kv_last_error().decode())


# The handle of the current stream without a Stream object around it: a call's whole marshalling takes 3.4 us, and building
# the object took 2.8 more (a decode step of nine layers, call by call: 202 us of host work before, 148 after).  Asked
# anew by every call, as current_stream() would be; a torch without the function gets the object.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _dev(t, dtype, name):
    if t is None:
        return None
    if t.dtype != dtype or not t.is_cuda or not t.is_contiguous():
        raise TypeError(f"{name}: need a contiguous {dtype} tensor on the GPU, got {t.dtype} on {t.device}")
    return t.data_ptr()


def make_spec(num_layers, num_q_heads, num_kv_heads, k_dim, v_dim=None, v_aliases_k=False, block_tokens=256,
              param_format=PARAMS_F16):
    return Spec(num_layers, num_q_heads, num_kv_heads, k_dim, k_dim if v_dim is None else v_dim,
                1 if v_aliases_k else 0, block_tokens, 64, param_format)


class Pool:
    """Device arrays of one paged Q4 pool: [layers][blocks][kv_heads][256][dim/8 | dim/64]."""

    def __init__(self, spec, dim, num_blocks, device="cuda", poison=False):
        shp = (spec.num_layers, num_blocks, spec.num_kv_heads, spec.block_tokens)
        self.dim, self.num_blocks, self.extent = dim, num_blocks, (spec.num_layers, spec.num_kv_heads, dim)
        # torch has no uint32/uint16 arithmetic, and none is needed: int32 / int16 storage of the same bits
        self.codes = torch.zeros(shp + (dim // 8,), dtype=torch.int32, device=device)
        self.scale = torch.zeros(shp + (dim // 64,), dtype=torch.int16, device=device)
        self.bias = torch.zeros(shp + (dim // 64,), dtype=torch.int16, device=device)
        if poison:                      # every slot decodes to NaN until it is written
            nan_bits = 0x7FC0 if spec.param_format == PARAMS_BF16 else 0x7E00
            self.codes.fill_(-1)
            self.scale.fill_(nan_bits)
            self.bias.fill_(nan_bits)

    @classmethod
    def of(cls, codes, scale, bias):
        """A pool around arrays that the caller has: int32 codes, int16 bits of scale and bias, shaped as above."""
        lead = tuple(codes.shape[:-1])
        if not (codes.dim() == 5 and tuple(scale.shape[:-1]) == lead == tuple(bias.shape[:-1]) and
                scale.shape[-1] * 8 == codes.shape[-1] == bias.shape[-1] * 8):
            raise ValueError(f"codes {tuple(codes.shape)}, scale {tuple(scale.shape)} and bias {tuple(bias.shape)} are no pool")
        for t, kind, name in ((codes, torch.int32, "codes"), (scale, torch.int16, "scale"), (bias, torch.int16, "bias")):
            _dev(t, kind, name)
        p = cls.__new__(cls)
        p.dim, p.num_blocks, p.codes, p.scale, p.bias = codes.shape[-1] * 8, codes.shape[1], codes, scale, bias
        p.extent = (lead[0], lead[2], p.dim) if lead[3] == 256 else None
        return p

    def c(self):
        return _CPool(self.codes.data_ptr(), self.scale.data_ptr(), self.bias.data_ptr(), self.num_blocks)


class HeadForm:
    """q4kv_head_form: what happens to a head of Q and K before it is used.  q_weight / k_weight: float32
    [layers of the call][norm_dim] on the GPU or None; cos / sin: float32 [positions][rot_dim / 2] on the GPU or None."""

    def __init__(self, norm_dim=0, q_weight=None, k_weight=None, eps=1e-6, rot_begin=0, rot_dim=0, neighbours=False, cos=None,
                 sin=None):
        self.norm_dim, self.q_weight, self.k_weight, self.eps = norm_dim, q_weight, k_weight, eps
        self.rot_begin, self.rot_dim, self.neighbours, self.cos, self.sin = rot_begin, rot_dim, neighbours, cos, sin

    def c(self, layers):
        # everything is asked on every call: a tensor may change its shape, type or place (resize_, set_, .data) in between
        q_weight, k_weight, cos, sin, table_len = self.q_weight, self.k_weight, self.cos, self.sin, 0
        rows = layers, self.norm_dim
        if q_weight is not None and q_weight.shape != rows:
            raise ValueError(f"q_weight: {tuple(q_weight.shape)} instead of {rows}")
        if k_weight is not None and k_weight.shape != rows:
            raise ValueError(f"k_weight: {tuple(k_weight.shape)} instead of {rows}")
        if self.rot_dim:
            table = () if cos is None or sin is None else cos.shape
            if len(table) != 2 or table[1] * 2 != self.rot_dim or sin.shape != table:
                raise ValueError(f"cos and sin: one shape, [positions][{self.rot_dim // 2}]")
            table_len = table[0]
        f32 = torch.float32
        return _CHeadForm(_dev(q_weight, f32, "q_weight"), _dev(k_weight, f32, "k_weight"), _dev(cos, f32, "cos"), _dev(sin, f32, "sin"),
                          self.norm_dim, self.eps, self.rot_begin, self.rot_dim, 1 if self.neighbours else 0, table_len)


class BlockTables:
    """q4kv_tables: block table [agents][max_blocks], lengths [agents] and counts [blocks], int32 on the GPU.  refused: int32 [1], how
    many rows the last call could not serve."""

    def __init__(self, num_agents, max_blocks, num_blocks, device="cuda"):
        self._around(torch.full((num_agents, max_blocks), -1, dtype=torch.int32, device=device),
                     torch.zeros(num_agents, dtype=torch.int32, device=device), torch.zeros(num_blocks, dtype=torch.int32, device=device))

    @classmethod
    def of(cls, block_table, seq_len, refs):
        """Around arrays that the caller has."""
        t = cls.__new__(cls)
        t._around(block_table, seq_len, refs)
        return t

    def _around(self, block_table, seq_len, refs):
        self.block_table, self.seq_len, self.refs = block_table, seq_len, refs
        self.refused = torch.zeros(1, dtype=torch.int32, device=refs.device)

    def c(self):
        table, i32 = self.block_table, torch.int32
        if table.dim() != 2 or self.seq_len.numel() != table.shape[0]:
            raise ValueError(f"a table of {tuple(table.shape)} for {self.seq_len.numel()} lengths")
        return _CTables(_dev(table, i32, "block_table"), _dev(self.seq_len, i32, "seq_len"), _dev(self.refs, i32, "refs"),
                        _dev(self.refused, i32, "refused"), table.shape[0], table.shape[1], self.refs.numel())


class TokenMap:
    """What q4kv_resize_tables writes for the tokens that rows got longer by: begin int32 [agents + 1]; slot, agent and position
    int32 [max_tokens], -1 behind the last token."""

    def __init__(self, tables, max_tokens):
        device = tables.refs.device
        self.begin = torch.zeros(tables.block_table.shape[0] + 1, dtype=torch.int32, device=device)
        self.slot, self.agent, self.position = (torch.full((max_tokens,), -1, dtype=torch.int32, device=device) for _ in range(3))


class BeamChoice:
    """What q4kv_beam_select writes: parent and token int32, score float32, all [groups][num_out]."""

    def __init__(self, groups, num_out, device="cuda"):
        self.parent, self.token = (torch.empty((groups, num_out), dtype=torch.int32, device=device) for _ in range(2))
        self.score = torch.empty((groups, num_out), dtype=torch.float32, device=device)


class BlockPool:
    """q4kv_block_pool: host-side bookkeeping of block ownership (Sec. 3.1).  Marshalling only."""
    ENOSPACE = -6

    def __init__(self, num_blocks):
        self._h = lib().q4kv_block_pool_create(num_blocks)
        if not self._h:
            raise ValueError("q4kv_block_pool_create failed")

    def close(self):
        if self._h:
            lib().q4kv_block_pool_destroy(self._h)
            self._h = None

    def __del__(self):
        self.close()

    @staticmethod
    def _ok(rc):
        if rc < 0:
            raise Q4KVError(rc, "block pool: " + {-1: "bad argument or unknown agent", -3: "more blocks than the row holds",
                                                  -6: "not enough free blocks"}.get(rc, "error"))
        return rc

    def reserve(self, agent_id, tokens):
        return self._ok(lib().q4kv_block_pool_reserve(self._h, agent_id, tokens))

    def release(self, agent_id):
        return self._ok(lib().q4kv_block_pool_release(self._h, agent_id))

    def blocks(self, agent_id):
        n = self._ok(lib().q4kv_block_pool_blocks(self._h, agent_id, None, 0))
        ids = (C.c_int32 * max(n, 1))()
        self._ok(lib().q4kv_block_pool_blocks(self._h, agent_id, ids, n))
        return list(ids[:n])

    def table_row(self, agent_id, max_blocks, fill=-1):
        row = (C.c_int32 * max_blocks)()
        self._ok(lib().q4kv_block_pool_table_row(self._h, agent_id, row, max_blocks, fill))
        return list(row)

    def touch(self, agent_id):
        self._ok(lib().q4kv_block_pool_touch(self._h, agent_id))

    def pin(self, agent_id, pinned=True):
        self._ok(lib().q4kv_block_pool_pin(self._h, agent_id, 1 if pinned else 0))

    def lru_victim(self):
        return lib().q4kv_block_pool_lru_victim(self._h)

    def free_blocks(self):
        return lib().q4kv_block_pool_free_blocks(self._h)

    def owner(self, block_id):
        return lib().q4kv_block_pool_owner(self._h, block_id)

    def fork(self, parent_id, child_id, tokens):
        """The pairs (source block, destination block) that q4kv_copy_blocks is to copy: none or one."""
        return self._with_pair(lib().q4kv_block_pool_fork, parent_id, child_id, tokens)

    def truncate(self, agent_id, tokens):
        """As fork()."""
        return self._with_pair(lib().q4kv_block_pool_truncate, agent_id, tokens)

    def _with_pair(self, call, *args):
        src, dst = C.c_int32(-1), C.c_int32(-1)
        self._ok(call(self._h, *args, C.byref(src), C.byref(dst)))
        return [] if dst.value < 0 else [(src.value, dst.value)]

    def compact(self):
        """The pairs that one call of q4kv_copy_blocks is to copy before any block is used again."""
        cap = lib().q4kv_block_pool_compact(self._h, None, None, 0)
        while self._ok(cap) > 0:
            src, dst = (C.c_int32 * cap)(), (C.c_int32 * cap)()
            n = lib().q4kv_block_pool_compact(self._h, src, dst, cap)
            if n != -3:                       # else another thread has freed blocks in between: more to move
                return list(zip(src, dst))[:self._ok(n)]
            cap = lib().q4kv_block_pool_compact(self._h, None, None, 0)
        return []

    def shares(self, block_id):
        return self._ok(lib().q4kv_block_pool_shares(self._h, block_id))


def q4kv_version():
    return lib().q4kv_version()


def q4kv_cache_bytes(spec, tokens):
    r = lib().q4kv_cache_bytes(C.byref(spec), tokens)
    if r < 0:
        _check(-1)
    return r


def q4kv_block_image_bytes(spec, num_blocks):
    return lib().q4kv_block_image_bytes(C.byref(spec), num_blocks)


def _image_call(fn, spec, kpool, vpool, block_ids, image):
    """block_ids: int32 tensor on the GPU; image: uint8 tensor on the GPU or in pinned host memory."""
    if not (image.dtype == torch.uint8 and image.is_contiguous() and (image.is_cuda or image.is_pinned())):
        raise ValueError("image: contiguous uint8 tensor on the GPU or in pinned host memory")
    kp = kpool.c()
    vp = None if spec.v_aliases_k else vpool.c()
    _check(fn(C.byref(spec), C.byref(kp), None if vp is None else C.byref(vp), _dev(block_ids, torch.int32, "block_ids"),
              block_ids.numel(), image.data_ptr(), image.numel(), _stream()))


def q4kv_export_blocks(spec, kpool, vpool, block_ids, image=None):
    """Gather the listed blocks of every layer into a block image (see include/q4kv.h); returns the image."""
    if image is None:
        image = torch.empty(q4kv_block_image_bytes(spec, block_ids.numel()), dtype=torch.uint8, device=block_ids.device)
    _image_call(lib().q4kv_export_blocks, spec, kpool, vpool, block_ids, image)
    return image


def q4kv_import_blocks(spec, kpool, vpool, block_ids, image):
    """Scatter a block image into the listed blocks of every layer."""
    _image_call(lib().q4kv_import_blocks, spec, kpool, vpool, block_ids, image)


def q4kv_read_probe(buf, sink):
    """Measurement helper: read the contiguous GPU tensor `buf` once (nothing is written); sink: int32 [1] on the GPU."""
    if not (buf.is_cuda and buf.is_contiguous() and sink.is_cuda and sink.numel() >= 1 and sink.element_size() == 4):
        raise ValueError("q4kv_read_probe: contiguous GPU tensors, sink of at least one 4-byte element")
    _check(lib().q4kv_read_probe(buf.data_ptr(), buf.numel() * buf.element_size(), sink.data_ptr(),
                                 _stream()))


def q4kv_quantize(x, codes=None, scale=None, bias=None, param_format=None):
    """x: fp16 [..., dim] on the GPU -> (codes int32 [..., dim/8], scale int16 [..., dim/64], bias same).
    param_format None: q4kv_quantize; PARAMS_F16 / PARAMS_BF16: q4kv_quantize_fmt."""
    dim = x.shape[-1]
    rows = x.numel() // dim if dim else 0
    lead = tuple(x.shape[:-1])
    if codes is None:
        codes = torch.empty(lead + (dim // 8,), dtype=torch.int32, device=x.device)
        scale = torch.empty(lead + (dim // 64,), dtype=torch.int16, device=x.device)
        bias = torch.empty(lead + (dim // 64,), dtype=torch.int16, device=x.device)
    outs = (_dev(codes, torch.int32, "codes"), _dev(scale, torch.int16, "scale"), _dev(bias, torch.int16, "bias"))
    if param_format is None:
        _check(lib().q4kv_quantize(_dev(x, torch.float16, "x"), rows, dim, *outs, _stream()))
    else:
        _check(lib().q4kv_quantize_fmt(_dev(x, torch.float16, "x"), rows, dim, int(param_format), *outs, _stream()))
    return codes, scale, bias


def q4kv_dequantize(codes, scale, bias, out=None, param_format=None):
    dim = codes.shape[-1] * 8
    rows = codes.numel() // codes.shape[-1] if codes.shape[-1] else 0
    if out is None:
        out = torch.empty(tuple(codes.shape[:-1]) + (dim,), dtype=torch.float16, device=codes.device)
    ins = (_dev(codes, torch.int32, "codes"), _dev(scale, torch.int16, "scale"), _dev(bias, torch.int16, "bias"))
    if param_format is None:
        _check(lib().q4kv_dequantize(*ins, rows, dim, _dev(out, torch.float16, "out"), _stream()))
    else:
        _check(lib().q4kv_dequantize_fmt(*ins, rows, dim, int(param_format), _dev(out, torch.float16, "out"), _stream()))
    return out


def q4kv_append(spec, kpool, vpool, k_new, v_new, block_table, seq_len_before, layer_begin=0, layer_end=None):
    """k_new / v_new: fp16 [layers_in_call][A][C][kv_heads][dim]; block_table int32 [A][max_blocks] (device)."""
    layer_end = spec.num_layers if layer_end is None else layer_end
    A, Cn = k_new.shape[1], k_new.shape[2]
    kp = kpool.c()
    vp = None if spec.v_aliases_k else vpool.c()
    _check(lib().q4kv_append(C.byref(spec), C.byref(kp), None if vp is None else C.byref(vp),
                             _dev(k_new, torch.float16, "k_new"), _dev(v_new, torch.float16, "v_new"),
                             _dev(block_table, torch.int32, "block_table"), block_table.shape[1],
                             _dev(seq_len_before, torch.int32, "seq_len_before"), A, Cn, layer_begin, layer_end,
                             _stream()))


def _pools(spec, kpool, vpool):
    """The pools of a call as the library takes them, refused where their arrays are not those of the spec."""
    if kpool.extent != (spec.num_layers, spec.num_kv_heads, spec.k_dim):
        raise ValueError(f"K pool of (layers, KV heads, width) {kpool.extent}, not {(spec.num_layers, spec.num_kv_heads, spec.k_dim)}")
    if spec.v_aliases_k:
        return C.byref(kpool.c()), None
    if vpool is not None and vpool.extent != (spec.num_layers, spec.num_kv_heads, spec.v_dim):
        raise ValueError(f"V pool of (layers, KV heads, width) {vpool.extent}, not {(spec.num_layers, spec.num_kv_heads, spec.v_dim)}")
    return C.byref(kpool.c()), None if vpool is None else C.byref(vpool.c())


def _token_rows(t, heads, dim, name):
    """[layers][agents][chunk][heads][dim] with contiguous tokens a fixed stride apart -> that stride in elements."""
    shape = t.shape
    if len(shape) != 5 or shape[3] != heads or shape[4] != dim or not t.is_cuda:
        raise TypeError(f"{name}: need [layers][agents][chunk][{heads}][{dim}] on the GPU, got {tuple(shape)} on {t.device}")
    s0, s1, s2, s3, s4 = t.stride()
    if 0 in shape[:3]:                    # no tokens: nothing is a stride apart
        return heads * dim
    # the stride of an axis of one element means nothing: the last axis that has more gives the distance of two tokens
    stride, rows = None, 1
    for size, step in ((shape[2], s2), (shape[1], s1), (shape[0], s0)):
        if size > 1:
            if stride is None and step % rows == 0:
                stride = step // rows
            if stride is None or step != stride * rows:
                raise TypeError(f"{name}: tokens are not a fixed stride apart (strides {t.stride()})")
        rows *= size
    if (dim > 1 and s4 != 1) or (heads > 1 and s3 != dim):
        raise TypeError(f"{name}: the heads of a token must be contiguous (strides {t.stride()})")
    return heads * dim if stride is None else stride


def q4kv_norm_rope_append(spec, kpool, vpool, form, q, k_new, v_new, block_table, seq_len_before, positions=None,
                          layer_begin=0, layer_end=None, q_out=None):
    """q / k_new / v_new: fp16 or bf16 [layers_in_call][A][C][heads][dim], possibly parts of one fused projection (tokens a fixed
    stride apart); form: HeadForm.  Returns the prepared queries, fp16 [layers_in_call][A][C][q_heads][k_dim]."""
    layer_end = spec.num_layers if layer_end is None else layer_end
    hq, hkv, dk = spec.num_q_heads, spec.num_kv_heads, spec.k_dim
    q_stride, k_stride, v_stride = _token_rows(q, hq, dk, "q"), _token_rows(k_new, hkv, dk, "k_new"), 0
    if v_new is not None:
        v_stride = _token_rows(v_new, hkv, spec.v_dim, "v_new")
    kind, lead = q.dtype, q.shape[:3]
    if kind not in (torch.float16, torch.bfloat16) or k_new.dtype != kind or (v_new is not None and v_new.dtype != kind):
        raise TypeError(f"q, k_new and v_new: fp16 or bf16, all of one type, got {kind}, {k_new.dtype}")
    if k_new.shape[:3] != lead or (v_new is not None and v_new.shape[:3] != lead):
        raise TypeError(f"q, k_new and v_new differ in layers, agents or tokens: {tuple(lead)}, {tuple(k_new.shape[:3])}")
    Lr, A, Cn = lead
    if Lr != layer_end - layer_begin:
        raise ValueError(f"{Lr} layers of projections for {layer_end - layer_begin} layers")
    if q_out is None:
        q_out = torch.empty((Lr, A, Cn, hq, dk), dtype=torch.float16, device=q.device)
    elif q_out.shape != (Lr, A, Cn, hq, dk):
        raise ValueError(f"q_out: {tuple(q_out.shape)} instead of {(Lr, A, Cn, hq, dk)}")
    if block_table.shape[0] != A or seq_len_before.numel() != A:
        raise ValueError(f"{A} agents, {block_table.shape[0]} rows of blocks, {seq_len_before.numel()} lengths")
    if positions is not None and tuple(positions.shape) != (A, Cn):
        raise ValueError(f"positions: {tuple(positions.shape)} instead of {(A, Cn)}")
    kp, vp = _pools(spec, kpool, vpool)
    _check(lib().q4kv_norm_rope_append(
        C.byref(spec), kp, vp, C.byref(form.c(Lr)), q.data_ptr(),
        k_new.data_ptr(), None if v_new is None else v_new.data_ptr(), 1 if kind == torch.bfloat16 else 0, q_stride, k_stride,
        v_stride, _dev(q_out, torch.float16, "q_out"), _dev(block_table, torch.int32, "block_table"), block_table.shape[1],
        _dev(seq_len_before, torch.int32, "seq_len_before"), _dev(positions, torch.int32, "positions"), A, Cn, layer_begin,
        layer_end, _stream()))
    return q_out


def _slot_rows(t, heads, dim, name):
    """[layers][tokens][heads][dim] -> the stride of its tokens, as _token_rows; most tensors are told by their strides alone."""
    if t.dim() != 4:
        raise TypeError(f"{name}: need [layers][tokens][{heads}][{dim}], got {tuple(t.shape)}")
    layers, tokens, h, d = t.shape
    s0, s1, s2, s3 = t.stride()
    if h == heads and d == dim and s3 == 1 and s2 == dim and tokens > 1 and (layers == 1 or s0 == s1 * tokens) and t.is_cuda:
        return s1
    return _token_rows(t.unsqueeze(1), heads, dim, name)


def q4kv_append_slots(spec, kpool, vpool, k_new, v_new, slot, layer_begin=0, layer_end=None):
    """k_new / v_new: fp16 or bf16 [layers_in_call][tokens][kv_heads][dim], possibly parts of one fused projection (tokens a fixed
    stride apart); slot: int32 [tokens] on the GPU, block * 256 + place, outside the pool: the token is skipped."""
    layer_end = spec.num_layers if layer_end is None else layer_end
    hkv, kind, lead, v_stride = spec.num_kv_heads, k_new.dtype, k_new.shape[:2], 0
    k_stride = _slot_rows(k_new, hkv, spec.k_dim, "k_new")
    if v_new is not None:
        v_stride = _slot_rows(v_new, hkv, spec.v_dim, "v_new")
    if kind not in (torch.float16, torch.bfloat16) or (v_new is not None and v_new.dtype != kind):
        raise TypeError(f"k_new and v_new: fp16 or bf16, both of one type, got {kind}")
    if v_new is not None and v_new.shape[:2] != lead:
        raise TypeError(f"k_new and v_new differ in layers or tokens: {tuple(lead)}, {tuple(v_new.shape[:2])}")
    if lead[0] != layer_end - layer_begin:
        raise ValueError(f"{lead[0]} layers of rows for {layer_end - layer_begin} layers")
    if slot.numel() != lead[1]:
        raise ValueError(f"{slot.numel()} slots for {lead[1]} tokens")
    kp, vp = _pools(spec, kpool, vpool)
    _check(lib().q4kv_append_slots(C.byref(spec), kp, vp, k_new.data_ptr(), None if v_new is None else v_new.data_ptr(),
                                   1 if kind == torch.bfloat16 else 0, k_stride, v_stride, _dev(slot, torch.int32, "slot"), lead[1],
                                   layer_begin, layer_end, _stream()))


def q4kv_tables_workspace(tables):
    """The workspace that q4kv_beam_reorder needs, and q4kv_resize_tables with pools."""
    return torch.empty(lib().q4kv_tables_workspace_bytes(tables.block_table.shape[0]), dtype=torch.uint8, device=tables.refs.device)


def q4kv_resize_tables(tables, new_len, out=None, spec=None, kpool=None, vpool=None, workspace=None):
    """The agents' lengths become new_len (int32 [agents] on the GPU).  out: a TokenMap to fill, or None.  spec and pools: blocks
    that are shared where a row goes on or is cut are copied; None: see include/q4kv.h."""
    t, kp, vp = tables.c(), None, None
    if new_len.numel() != t.num_agents:
        raise ValueError(f"{new_len.numel()} lengths for {t.num_agents} agents")
    if spec is not None:
        kp, vp = _pools(spec, kpool, vpool)
        if workspace is None:
            workspace = q4kv_tables_workspace(tables)
    places, begin, slot, agent, position = 0, None, None, None, None
    if out is not None:
        i32 = torch.int32
        places, begin, slot = out.slot.numel(), _dev(out.begin, i32, "begin"), _dev(out.slot, i32, "slot")
        agent, position = _dev(out.agent, i32, "agent"), _dev(out.position, i32, "position")
        if out.begin.numel() != t.num_agents + 1 or any(x is not None and x.numel() != places for x in (out.agent, out.position)):
            raise ValueError("out: a map of other tables, or of arrays of different lengths")
    _check(lib().q4kv_resize_tables(C.byref(t), _dev(new_len, torch.int32, "new_len"), places, begin, slot, agent, position,
                                    None if spec is None else C.byref(spec), kp, vp, _dev(workspace, torch.uint8, "workspace"),
                                    0 if workspace is None else workspace.numel(), _stream()))
    return out


def q4kv_beam_reorder(spec, kpool, vpool, tables, parent, workspace=None):
    """Row i of the tables becomes what row parent[i] was (int32 [agents] on the GPU, outside: an empty row)."""
    t = tables.c()
    if parent.numel() != t.num_agents:
        raise ValueError(f"{parent.numel()} parents for {t.num_agents} agents")
    if workspace is None:
        workspace = q4kv_tables_workspace(tables)
    kp, vp = _pools(spec, kpool, vpool)
    _check(lib().q4kv_beam_reorder(C.byref(spec), kp, vp, C.byref(t), _dev(parent, torch.int32, "parent"),
                                   _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream()))


_LOGITS = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}


def q4kv_beam_select_workspace(logits, num_out):
    """The workspace of q4kv_beam_select for rows like these."""
    rows, vocab = logits.shape
    need = lib().q4kv_beam_select_workspace_bytes(_LOGITS[logits.dtype], vocab, rows, num_out)
    if need == 0:
        raise ValueError(lib().q4kv_last_error().decode())
    return torch.empty(need, dtype=torch.uint8, device=logits.device)


def q4kv_beam_select(logits, score, group_begin, num_out, end_token=None, out=None, workspace=None):
    """logits: fp16, bf16 or fp32 [agents][vocab], rows any stride apart; score: float32 [agents]; group_begin: int32 [groups + 1];
    end_token: int32 [agents] or None.  Returns a BeamChoice (out, if given)."""
    if logits.dim() != 2 or logits.dtype not in _LOGITS or not logits.is_cuda or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise TypeError(f"logits: need [agents][vocab] of fp16, bf16 or fp32 with contiguous rows on the GPU, got {logits.dtype} {tuple(logits.shape)}")
    rows, vocab = logits.shape
    groups = group_begin.numel() - 1
    if groups < 0 or score.numel() != rows or (end_token is not None and end_token.numel() != rows):
        raise ValueError(f"{rows} rows of logits, {score.numel()} scores, {group_begin.numel()} bounds")
    if out is None:
        out = BeamChoice(groups, num_out, logits.device)
    elif out.parent.shape != (groups, num_out) or out.token.shape != (groups, num_out) or out.score.shape != (groups, num_out):
        raise ValueError(f"out: {tuple(out.parent.shape)} instead of {(groups, num_out)}")
    if workspace is None:
        workspace = q4kv_beam_select_workspace(logits, num_out)
    i32, f32 = torch.int32, torch.float32
    _check(lib().q4kv_beam_select(logits.data_ptr(), _LOGITS[logits.dtype], logits.stride(0) if rows > 1 else vocab, vocab, rows,
                                  _dev(score, f32, "score"), _dev(end_token, i32, "end_token"), _dev(group_begin, i32, "group_begin"),
                                  groups, num_out, _dev(out.parent, i32, "parent"), _dev(out.token, i32, "token"),
                                  _dev(out.score, f32, "score"), _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream()))
    return out


def q4kv_copy_blocks(spec, kpool, vpool, src_ids, dst_ids):
    """Block dst_ids[i] becomes a copy of block src_ids[i], every layer, K and V; ids: int32 tensors on the GPU."""
    if src_ids.numel() != dst_ids.numel():
        raise ValueError(f"{src_ids.numel()} sources for {dst_ids.numel()} destinations")
    kp, vp = _pools(spec, kpool, vpool)
    _check(lib().q4kv_copy_blocks(C.byref(spec), kp, vp, _dev(src_ids, torch.int32, "src_ids"), _dev(dst_ids, torch.int32, "dst_ids"),
                                  src_ids.numel(), _stream()))


def q4kv_default_split_tokens(spec, num_agents, q_len, max_seq_len, layers_in_call):
    return lib().q4kv_default_split_tokens(C.byref(spec), num_agents, q_len, max_seq_len, layers_in_call)


def q4kv_attention_workspace_bytes(spec, num_agents, q_len, max_seq_len, split_tokens, layers_in_call):
    return lib().q4kv_attention_workspace_bytes(C.byref(spec), num_agents, q_len, max_seq_len, split_tokens,
                                                layers_in_call)


def q4kv_batched_attention(spec, kpool, vpool, q, block_table, seq_len, max_seq_len, sm_scale, window=0,
                           split_tokens=0, layer_begin=0, layer_end=None, out=None, workspace=None):
    """q: fp16 [layers_in_call][A][q_len][q_heads][k_dim] -> fp16 out of the same leading shape, v_dim wide.
    window: one int for all layers, or a sequence with one window per layer of the call (q4kv_batched_attention_windows).
    workspace: uint8 tensor on the GPU; None allocates what a decode call needs and nothing for q_len > 1.  A chunk call
    shares few or ragged agents out over the whole chip if it is given one of exactly q4kv_attention_workspace_bytes(...)
    bytes (up to 136 MB); without, its results are bit-identical to q4kv_batched_attention_static's."""
    layer_end = spec.num_layers if layer_end is None else layer_end
    Lr, A, q_len = q.shape[0], q.shape[1], q.shape[2]
    if out is None:
        out = torch.empty((Lr, A, q_len, spec.num_q_heads, spec.v_dim), dtype=torch.float16, device=q.device)
    if workspace is None:
        need = q4kv_attention_workspace_bytes(spec, max(A, 1), q_len, max_seq_len, split_tokens, max(Lr, 1)) if q_len == 1 else 0
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    kp = kpool.c()
    vp = None if spec.v_aliases_k else vpool.c()
    common = (C.byref(spec), C.byref(kp), None if vp is None else C.byref(vp),
              _dev(q, torch.float16, "q"), _dev(out, torch.float16, "out"),
              _dev(block_table, torch.int32, "block_table"), block_table.shape[1],
              _dev(seq_len, torch.int32, "seq_len"), A, q_len, max_seq_len, float(sm_scale))
    tail = (int(split_tokens), layer_begin, layer_end, workspace.data_ptr(), workspace.numel(), _stream())
    if isinstance(window, (list, tuple)) or hasattr(window, "__len__"):      # one window per layer of the call (host)
        if len(window) != layer_end - layer_begin:
            raise ValueError(f"{len(window)} windows for {layer_end - layer_begin} layers")
        windows = (C.c_int32 * len(window))(*[int(x) for x in window])
        _check(lib().q4kv_batched_attention_windows(*common, windows, *tail))
    else:
        _check(lib().q4kv_batched_attention(*common, int(window), *tail))
    return out


def q4kv_shared_prefix_workspace_bytes(spec, num_agents, max_seq_len, layers_in_call):
    return lib().q4kv_shared_prefix_workspace_bytes(C.byref(spec), num_agents, max_seq_len, layers_in_call)


def q4kv_shared_prefix_attention(spec, kpool, vpool, q, block_table, seq_len, group_begin, prefix_len, max_seq_len, sm_scale,
                                 layer_begin=0, layer_end=None, out=None, workspace=None):
    """Decode attention of agents in groups that share a prefix: q fp16 [layers_in_call][A][1][q_heads][k_dim]; group_begin int32
    [groups + 1] and prefix_len int32 [groups] on the GPU (both None: nobody shares).  workspace: uint8 tensor on the GPU of
    q4kv_shared_prefix_workspace_bytes(...) bytes, or None: allocated."""
    layer_end = spec.num_layers if layer_end is None else layer_end
    Lr, A = q.shape[0], q.shape[1]
    if q.shape[2] != 1:
        raise ValueError(f"{q.shape[2]} query tokens per agent: this is a decode call")
    groups = 0 if prefix_len is None else prefix_len.numel()
    if groups and (group_begin is None or group_begin.numel() != groups + 1):
        raise ValueError(f"{groups} groups need {groups + 1} bounds")
    if q.shape[3] != spec.num_q_heads or q.shape[4] != spec.k_dim or Lr != layer_end - layer_begin:
        raise ValueError(f"q: {tuple(q.shape)} for {layer_end - layer_begin} layers of {spec.num_q_heads} heads, {spec.k_dim} wide")
    if block_table.shape[0] != A or seq_len.numel() != A:
        raise ValueError(f"{A} agents, {block_table.shape[0]} rows of blocks, {seq_len.numel()} lengths")
    if out is None:
        out = torch.empty((Lr, A, 1, spec.num_q_heads, spec.v_dim), dtype=torch.float16, device=q.device)
    elif out.shape != (Lr, A, 1, spec.num_q_heads, spec.v_dim):
        raise ValueError(f"out: {tuple(out.shape)} instead of {(Lr, A, 1, spec.num_q_heads, spec.v_dim)}")
    if workspace is None:
        need = q4kv_shared_prefix_workspace_bytes(spec, max(A, 1), max_seq_len, max(Lr, 1))
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    kp, vp = _pools(spec, kpool, vpool)
    _check(lib().q4kv_shared_prefix_attention(
        C.byref(spec), kp, vp, _dev(q, torch.float16, "q"),
        _dev(out, torch.float16, "out"), _dev(block_table, torch.int32, "block_table"), block_table.shape[1],
        _dev(seq_len, torch.int32, "seq_len"), A, _dev(group_begin, torch.int32, "group_begin"),
        _dev(prefix_len, torch.int32, "prefix_len"), groups, max_seq_len, float(sm_scale), layer_begin, layer_end,
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream()))
    return out


STATIC_SCRATCH_BYTES = 16 << 20   # Q4KV_STATIC_SCRATCH_BYTES


def q4kv_batched_attention_static(spec, kpool, vpool, q, out, block_table, seq_len, max_seq_len, sm_scale, window=0,
                                  split_tokens=0, layer_begin=0, layer_end=None):
    """q4kv_batched_attention_static: the decode path's workspace comes from the library's fixed per-GPU array.
    Allocates no tensor: `out` (fp16 [layers_in_call][A][q_len][q_heads][v_dim]) is the caller's."""
    layer_end = spec.num_layers if layer_end is None else layer_end
    kp = kpool.c()
    vp = None if spec.v_aliases_k else vpool.c()
    _check(lib().q4kv_batched_attention_static(
        C.byref(spec), C.byref(kp), None if vp is None else C.byref(vp), _dev(q, torch.float16, "q"),
        _dev(out, torch.float16, "out"), _dev(block_table, torch.int32, "block_table"), block_table.shape[1],
        _dev(seq_len, torch.int32, "seq_len"), q.shape[1], q.shape[2], max_seq_len, float(sm_scale), int(window),
        int(split_tokens), layer_begin, layer_end, _stream()))
    return out


def q4kv_decode_plan(spec, seq_len, max_seq_len, workspace, window=0, split_tokens=0, layers_in_call=1):
    """q4kv_decode_plan: prepare `workspace` (uint8 tensor on the GPU) for q4kv_batched_attention_planned calls."""
    _check(lib().q4kv_decode_plan(C.byref(spec), _dev(seq_len, torch.int32, "seq_len"), seq_len.numel(), max_seq_len,
                                  int(window), int(split_tokens), layers_in_call, workspace.data_ptr(),
                                  workspace.numel(), _stream()))


def q4kv_batched_attention_planned(spec, kpool, vpool, q, out, block_table, max_seq_len, sm_scale, workspace, window=0,
                                   split_tokens=0, layer_begin=0, layer_end=None):
    """q4kv_batched_attention_planned: decode attention (q_len 1) on a workspace prepared by q4kv_decode_plan."""
    layer_end = spec.num_layers if layer_end is None else layer_end
    kp = kpool.c()
    vp = None if spec.v_aliases_k else vpool.c()
    _check(lib().q4kv_batched_attention_planned(
        C.byref(spec), C.byref(kp), None if vp is None else C.byref(vp), _dev(q, torch.float16, "q"),
        _dev(out, torch.float16, "out"), _dev(block_table, torch.int32, "block_table"), block_table.shape[1], q.shape[1],
        max_seq_len, float(sm_scale), int(window), int(split_tokens), layer_begin, layer_end,
        workspace.data_ptr(), workspace.numel(), _stream()))
    return out
