"""Binding of libqsgd.so: the same entry points as include/qsgd.h, argument marshalling only. The calls
that a training loop makes every step go through the native module (csrc/python_binding.cpp), size
queries, plans and test hooks through ctypes. PyTorch supplies device memory and the CUDA stream; every
step of the path runs in the library's kernels. There is no CPU fallback: a missing library or a missing
device raises.
"""
import ctypes as C
import importlib.machinery
import importlib.util
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libqsgd.so")

NORM_L2, NORM_MAX = 0, 1
CODE_FIXED, CODE_ELIAS, CODE_ELIAS_DENSE = 0, 1, 2

DEV_CAPACITY, DEV_OVERRUN, DEV_POSITION, DEV_LEVEL, DEV_TABLE, DEV_TIMEOUT = 1, 2, 4, 8, 16, 32
DEV_PAGE = 64

TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}

EXPORTS = ["qsgd_message_capacity", "qsgd_workspace_bytes", "qsgd_fixed_layout", "qsgd_encode",
           "qsgd_decode_accumulate", "qsgd_sgd_step", "qsgd_decode_sgd_step",
           "qsgd_decode_accumulate_packed", "qsgd_decode_sgd_step_packed",
           "qsgd_status_string", "qsgd_launch_count", "qsgd_profile_enable",
           "qsgd_profile_kernel_count", "qsgd_profile_kernel_name", "qsgd_profile_collect",
           "qsgd_static_scratch_bytes", "qsgd_encode_elias_static",
           "qsgd_policy_plan_sizes", "qsgd_policy_plan", "qsgd_policy_message_capacity",
           "qsgd_policy_workspace_bytes", "qsgd_policy_encode", "qsgd_policy_decode_accumulate",
           "qsgd_policy_decode_sgd_step", "qsgd_test_set_wait_polls", "qsgd_test_default_wait_polls",
           "qsgd_set_launch_chaining", "qsgd_cache_page_bytes", "qsgd_cache_write", "qsgd_cache_read",
           "qsgd_cache_attend_workspace_bytes", "qsgd_cache_attend", "qsgd_quantize_rows", "qsgd_matmul_i8",
           "qsgd_linear_i8_workspace_bytes", "qsgd_linear_i8"]

_lib = None


class QsgdError(RuntimeError):
    pass


class PolicyStruct(C.Structure):
    """qsgd_policy of include/qsgd.h."""
    _fields_ = [("bucket_src", C.c_void_p), ("bucket_len", C.c_void_p), ("n_buckets", C.c_uint64),
                ("raw_src", C.c_void_p), ("raw_start", C.c_void_p), ("n_raw_segments", C.c_uint64),
                ("n_raw", C.c_uint64), ("n", C.c_uint64), ("quads", C.c_uint32)]


class CacheStruct(C.Structure):
    """qsgd_cache of include/qsgd.h."""
    _fields_ = [("data", C.c_void_p), ("n_pages", C.c_uint64), ("page_stride", C.c_uint64), ("head_stride", C.c_uint64),
                ("page_tokens", C.c_uint32), ("heads", C.c_uint32), ("head_dim", C.c_uint32), ("type", C.c_int)]


class CacheRowsStruct(C.Structure):
    """qsgd_cache_rows of include/qsgd.h."""
    _fields_ = [("table", C.c_void_p), ("table_stride", C.c_uint64), ("table_pages", C.c_uint32), ("sequences", C.c_uint32),
                ("lengths", C.c_void_p), ("starts", C.c_void_p), ("rows", C.c_uint64)]


def lib():
    """Loads libqsgd.so (must have been built: `python -m paper_1610_02132_b200.build`)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise QsgdError("libqsgd.so is not built; run paper_1610_02132_b200.build.build()")
        L = C.CDLL(_LIB_PATH)
        vp, u64, u32, sz = C.c_void_p, C.c_uint64, C.c_uint32, C.c_size_t
        L.qsgd_message_capacity.argtypes = [u64, u32, u32, C.c_int]
        L.qsgd_message_capacity.restype = sz
        L.qsgd_workspace_bytes.argtypes = [u64, u32, u32, C.c_int]
        L.qsgd_workspace_bytes.restype = sz
        L.qsgd_fixed_layout.argtypes = [u64, u32, u32, C.POINTER(u64)]
        L.qsgd_fixed_layout.restype = C.c_int
        L.qsgd_encode.argtypes = [vp, u64, u32, u32, C.c_int, C.c_int, u64, u32, u32, vp, sz, vp,
                                  vp, vp, vp]
        L.qsgd_encode.restype = C.c_int
        L.qsgd_decode_accumulate.argtypes = [C.POINTER(vp), C.POINTER(vp), C.POINTER(u64), u32, u64, u32, u32,
                                             C.c_int, vp, vp, vp]
        L.qsgd_decode_accumulate.restype = C.c_int
        L.qsgd_decode_accumulate_packed.argtypes = L.qsgd_decode_accumulate.argtypes
        L.qsgd_decode_accumulate_packed.restype = C.c_int
        L.qsgd_sgd_step.argtypes = [vp, vp, C.c_float, u32, u64, vp]
        L.qsgd_sgd_step.restype = C.c_int
        L.qsgd_decode_sgd_step.argtypes = [C.POINTER(vp), C.POINTER(vp), C.POINTER(u64), u32, u64, u32, u32,
                                           C.c_int, vp, C.c_float, vp, vp]
        L.qsgd_decode_sgd_step.restype = C.c_int
        L.qsgd_decode_sgd_step_packed.argtypes = L.qsgd_decode_sgd_step.argtypes
        L.qsgd_decode_sgd_step_packed.restype = C.c_int
        L.qsgd_status_string.argtypes = [C.c_int]
        L.qsgd_status_string.restype = C.c_char_p
        L.qsgd_static_scratch_bytes.argtypes = []
        L.qsgd_static_scratch_bytes.restype = sz
        L.qsgd_encode_elias_static.argtypes = [vp, u64, u32, u32, C.c_int, C.c_int, u64, u32, u32, vp,
                                               sz, vp, vp, vp]
        L.qsgd_encode_elias_static.restype = C.c_int
        L.qsgd_launch_count.argtypes = []
        L.qsgd_launch_count.restype = u64
        pu64, pu32, pp = C.POINTER(u64), C.POINTER(u32), C.POINTER(PolicyStruct)
        L.qsgd_policy_plan_sizes.argtypes = [pu64, u32, u32, u64, pu64, pu64, pu64]
        L.qsgd_policy_plan_sizes.restype = C.c_int
        L.qsgd_policy_plan.argtypes = [pu64, u32, u32, u64, pu64, pu32, pu64, pu64, pu32]
        L.qsgd_policy_plan.restype = C.c_int
        L.qsgd_policy_message_capacity.argtypes = [pp, u32, u32, C.c_int]
        L.qsgd_policy_message_capacity.restype = sz
        L.qsgd_policy_workspace_bytes.argtypes = [pp, u32, u32, C.c_int]
        L.qsgd_policy_workspace_bytes.restype = sz
        L.qsgd_policy_encode.argtypes = [vp, pp, u32, u32, C.c_int, C.c_int, u64, u32, u32, vp, sz, vp,
                                         vp, vp, vp]
        L.qsgd_policy_encode.restype = C.c_int
        L.qsgd_policy_decode_accumulate.argtypes = [C.POINTER(vp), C.POINTER(vp), pu64, u32, pp, u32, u32,
                                                    C.c_int, vp, vp, vp]
        L.qsgd_policy_decode_accumulate.restype = C.c_int
        L.qsgd_policy_decode_sgd_step.argtypes = [C.POINTER(vp), C.POINTER(vp), pu64, u32, pp, u32, u32,
                                                  C.c_int, vp, C.c_float, vp, vp]
        L.qsgd_policy_decode_sgd_step.restype = C.c_int
        pc, pr = C.POINTER(CacheStruct), C.POINTER(CacheRowsStruct)
        L.qsgd_cache_page_bytes.argtypes = [u32, u32, u32]
        L.qsgd_cache_page_bytes.restype = sz
        L.qsgd_cache_write.argtypes = [pc, pr, vp, u64, u64, vp, u64, u64, vp, vp]
        L.qsgd_cache_write.restype = C.c_int
        L.qsgd_cache_read.argtypes = L.qsgd_cache_write.argtypes
        L.qsgd_cache_read.restype = C.c_int
        L.qsgd_cache_attend_workspace_bytes.argtypes = [pc, u32]
        L.qsgd_cache_attend_workspace_bytes.restype = sz
        L.qsgd_cache_attend.argtypes = [pc, pr, vp, u64, u64, u32, C.c_float, vp, u64, u64, vp, vp, vp, vp]
        L.qsgd_cache_attend.restype = C.c_int
        L.qsgd_quantize_rows.argtypes = [vp, u64, u32, u64, C.c_int, vp, u64, vp, vp]
        L.qsgd_quantize_rows.restype = C.c_int
        L.qsgd_matmul_i8.argtypes = [vp, u64, vp, vp, u64, vp, vp, u64, u64, u32, vp, u64, C.c_int, vp, vp]
        L.qsgd_matmul_i8.restype = C.c_int
        L.qsgd_linear_i8_workspace_bytes.argtypes = [u64, u32]
        L.qsgd_linear_i8_workspace_bytes.restype = sz
        L.qsgd_linear_i8.argtypes = [vp, u64, C.c_int, vp, u64, vp, vp, u64, u64, u32, vp, u64, C.c_int, vp, vp, vp]
        L.qsgd_linear_i8.restype = C.c_int
        L.qsgd_set_launch_chaining.argtypes = [C.c_int]
        L.qsgd_set_launch_chaining.restype = C.c_int
        L.qsgd_test_set_wait_polls.argtypes = [u32]
        L.qsgd_test_set_wait_polls.restype = None
        L.qsgd_test_default_wait_polls.argtypes = []
        L.qsgd_test_default_wait_polls.restype = u32
        L.qsgd_profile_enable.argtypes = [C.c_int]
        L.qsgd_profile_enable.restype = None
        L.qsgd_profile_kernel_count.argtypes = []
        L.qsgd_profile_kernel_count.restype = C.c_int
        L.qsgd_profile_kernel_name.argtypes = [C.c_int]
        L.qsgd_profile_kernel_name.restype = C.c_char_p
        L.qsgd_profile_collect.argtypes = [C.POINTER(C.c_double), C.POINTER(u64)]
        L.qsgd_profile_collect.restype = C.c_int
        _lib = L
    return _lib


class _Native:
    """Stands in for the native module until the first call loads it."""

    def __getattr__(self, name):
        global _native
        from . import build
        path = build.native_path()
        if not os.path.exists(path):
            raise QsgdError("%s is not built; run paper_1610_02132_b200.build.build()" % os.path.basename(path))
        lib()                                             # the library it is linked against: its own message if missing
        loader = importlib.machinery.ExtensionFileLoader("_qsgd_native", path)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_qsgd_native", loader))
        loader.exec_module(module)
        module.set_error(QsgdError)
        _native = module
        return getattr(module, name)


_native = _Native()


def _check(st):
    if st != 0:
        raise QsgdError("qsgd status %d: %s" % (st, lib().qsgd_status_string(st).decode()))


def qsgd_message_capacity(n, bucket, s, code_kind):
    return int(lib().qsgd_message_capacity(n, bucket, s, code_kind))


def qsgd_workspace_bytes(n, bucket, s, code_kind):
    return int(lib().qsgd_workspace_bytes(n, bucket, s, code_kind))


def qsgd_fixed_layout(n, bucket, s):
    lay = (C.c_uint64 * 4)()
    _check(lib().qsgd_fixed_layout(n, bucket, s, lay))
    return [int(v) for v in lay]


def qsgd_launch_count():
    return int(lib().qsgd_launch_count())


def qsgd_set_launch_chaining(on):
    """Turns programmatic dependent launch of the library's kernels on or off; returns the previous setting."""
    return bool(lib().qsgd_set_launch_chaining(1 if on else 0))


def qsgd_test_set_wait_polls(polls):
    """Test hook: bound of the streaming encoder's main-loop waits (0 = give up at once)."""
    lib().qsgd_test_set_wait_polls(int(polls))


def qsgd_test_default_wait_polls():
    return int(lib().qsgd_test_default_wait_polls())


def qsgd_profile_enable(on):
    lib().qsgd_profile_enable(1 if on else 0)


def qsgd_profile_collect():
    """Returns {kernel name: (total ms, launches)} for the launches recorded since the last call."""
    L = lib()
    k = L.qsgd_profile_kernel_count()
    ms = (C.c_double * k)()
    cnt = (C.c_uint64 * k)()
    st = L.qsgd_profile_collect(ms, cnt)
    if st != 0:
        raise QsgdError("qsgd_profile_collect: cuda error %d" % st)
    return {L.qsgd_profile_kernel_name(i).decode(): (float(ms[i]), int(cnt[i]))
            for i in range(k) if cnt[i]}


def qsgd_encode(g, bucket, s, norm_kind, code_kind, seed, step, worker, out, out_bits,
                workspace=None, status_dev=None, stream=None, n=None):
    """Encode g (fp32 CUDA tensor) into `out` (uint8 CUDA tensor); see include/qsgd.h."""
    _check(_native.encode(g, n, bucket, s, norm_kind, code_kind, seed, step, worker, out, out_bits, workspace,
                          status_dev, stream))


def qsgd_static_scratch_bytes():
    return int(lib().qsgd_static_scratch_bytes())


def qsgd_encode_elias_static(g, bucket, s, norm_kind, code_kind, seed, step, worker, out, out_bits,
                             status_dev, stream=None):
    """Elias Encode without a workspace argument: the scratch is a 32 MiB array built into the
    library, so this call allocates nothing (for callers that may not allocate device memory when
    they encode). Same results as qsgd_encode; sizes beyond the built-in scratch raise. Calls
    that overlap on the GPU share the scratch and must be serialised by the caller."""
    _check(_native.encode_static(g, bucket, s, norm_kind, code_kind, seed, step, worker, out, out_bits, status_dev,
                                 stream))


def qsgd_decode_accumulate(msgs, tables, n, bucket, s, code_kind, acc, status_dev, stream=None,
                           payload_bytes=None):
    """acc <- ascending-k sum of the decoded messages; msgs / tables: lists of CUDA tensors
    (or raw device addresses); payload_bytes: optional list of payload lengths (read bound)."""
    _check(_native.decode(False, msgs, tables, payload_bytes, n, bucket, s, code_kind, acc, None, status_dev, stream))


def qsgd_decode_accumulate_packed(msgs, infos, n, bucket, s, code_kind, acc, status_dev, stream=None,
                                  msg_bytes=None):
    """As qsgd_decode_accumulate, for messages as Encode left them: infos[k] is the CUDA tensor (or
    device address) of message k's four info words; the tables are found on the device. msg_bytes
    defaults to the sizes of the message tensors."""
    _check(_native.decode(True, msgs, infos, msg_bytes, n, bucket, s, code_kind, acc, None, status_dev, stream))


def qsgd_decode_sgd_step_packed(msgs, infos, n, bucket, s, code_kind, x, eta, status_dev, stream=None,
                                msg_bytes=None):
    _check(_native.decode(True, msgs, infos, msg_bytes, n, bucket, s, code_kind, x, eta, status_dev, stream))


def qsgd_sgd_step(x, acc, eta, K, stream=None):
    _check(_native.sgd_step(x, acc, eta, K, stream))


def qsgd_decode_sgd_step(msgs, tables, n, bucket, s, code_kind, x, eta, status_dev, stream=None,
                         payload_bytes=None):
    _check(_native.decode(False, msgs, tables, payload_bytes, n, bucket, s, code_kind, x, eta, status_dev, stream))


# ------------------------------- per-tensor policy -------------------------------------------
class Policy:
    """A plan made by qsgd_policy_plan for tensors of the given sizes, with its arrays copied to
    the device (the copies are the only thing this class adds to the C calls)."""

    def __init__(self, tensor_sizes, bucket, min_quantized=10000, device="cuda"):
        T = len(tensor_sizes)
        sizes = (C.c_uint64 * max(T, 1))(*[int(m) for m in tensor_sizes])
        nb, ns, nr = C.c_uint64(), C.c_uint64(), C.c_uint64()
        _check(lib().qsgd_policy_plan_sizes(sizes, T, bucket, min_quantized, C.byref(nb), C.byref(ns), C.byref(nr)))
        nb, ns, nr = nb.value, ns.value, nr.value
        src = torch.zeros(max(nb, 1), dtype=torch.int64)
        ln = torch.zeros(max(nb, 1), dtype=torch.int32)
        rsrc = torch.zeros(max(ns, 1), dtype=torch.int64)
        rstart = torch.zeros(ns + 1, dtype=torch.int64)
        quads = C.c_uint32()
        as_p = lambda t, ct: C.cast(t.data_ptr(), C.POINTER(ct))
        _check(lib().qsgd_policy_plan(sizes, T, bucket, min_quantized, as_p(src, C.c_uint64), as_p(ln, C.c_uint32),
                                      as_p(rsrc, C.c_uint64), as_p(rstart, C.c_uint64), C.byref(quads)))
        self.bucket = bucket
        self.host = {"bucket_src": src[:nb], "bucket_len": ln[:nb], "raw_src": rsrc[:ns], "raw_start": rstart}
        self.dev = {k: v.to(device) for k, v in (("bucket_src", src), ("bucket_len", ln), ("raw_src", rsrc),
                                                ("raw_start", rstart))}
        self.n = int(sum(int(m) for m in tensor_sizes))
        self.n_buckets, self.n_raw_segments, self.n_raw, self.quads = nb, ns, nr, quads.value
        self.raw_prefix = (4 * nr + 15) // 16 * 16
        self.struct = PolicyStruct(self.dev["bucket_src"].data_ptr(), self.dev["bucket_len"].data_ptr(), nb,
                                   self.dev["raw_src"].data_ptr(), self.dev["raw_start"].data_ptr(), ns, nr,
                                   self.n, quads.value)


def qsgd_policy_message_capacity(plan, s, code_kind):
    return int(lib().qsgd_policy_message_capacity(C.byref(plan.struct), plan.bucket, s, code_kind))


def qsgd_policy_workspace_bytes(plan, s, code_kind):
    return int(lib().qsgd_policy_workspace_bytes(C.byref(plan.struct), plan.bucket, s, code_kind))


def _covered(t, name, plan):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous()):
        raise QsgdError("%s must be a contiguous CUDA tensor" % name)
    if t.numel() != plan.n:
        raise QsgdError("%s has %d elements, the plan covers %d" % (name, t.numel(), plan.n))


def qsgd_policy_encode(g, plan, s, norm_kind, code_kind, seed, step, worker, out, out_bits, workspace=None,
                       status_dev=None, stream=None):
    _covered(g, "g", plan)
    _check(_native.policy_encode(g, C.addressof(plan.struct), plan.bucket, s, norm_kind, code_kind, seed, step, worker, out,
                                 out_bits, workspace, status_dev, stream))


def qsgd_policy_decode_accumulate(msgs, tables, plan, s, code_kind, acc, status_dev, stream=None,
                                  payload_bytes=None):
    _covered(acc, "acc", plan)
    _check(_native.policy_decode(msgs, tables, payload_bytes, C.addressof(plan.struct), plan.bucket, s, code_kind, acc, None,
                                 status_dev, stream))


def qsgd_policy_decode_sgd_step(msgs, tables, plan, s, code_kind, x, eta, status_dev, stream=None,
                                payload_bytes=None):
    _covered(x, "x", plan)
    _check(_native.policy_decode(msgs, tables, payload_bytes, C.addressof(plan.struct), plan.bucket, s, code_kind, x, eta,
                                 status_dev, stream))


# ------------------------------- few-bit values outside the gradient exchange -----------------
def qsgd_cache_page_bytes(page_tokens, heads, head_dim):
    return int(lib().qsgd_cache_page_bytes(page_tokens, heads, head_dim))


class Cache:
    """A 4-bit cache of keys and values (qsgd_cache): its memory, [pages, heads, bytes of a page and head] in uint8, and what
    the calls have to know of it. `data` may be given: any strides, as long as the last dimension is contiguous."""

    def __init__(self, n_pages, page_tokens, heads, head_dim, dtype=torch.bfloat16, device="cuda", data=None):
        page = qsgd_cache_page_bytes(page_tokens, heads, head_dim)
        if not page or dtype not in (torch.float16, torch.bfloat16) or n_pages < 1:
            raise QsgdError("a cache has at least one page, of a multiple of 16 tokens, with heads of 64, 128, 192 or 256 "
                            "numbers in float16 or bfloat16")
        if data is None:
            data = torch.empty(n_pages, heads, page // heads, dtype=torch.uint8, device=device)
        if data.dtype != torch.uint8 or tuple(data.shape) != (n_pages, heads, page // heads) or data.stride(2) != 1:
            raise QsgdError("data must be uint8, [%d, %d, %d], contiguous along its last dimension" % (n_pages, heads, page // heads))
        self.data, self.dtype = data, dtype
        self.n_pages, self.page_tokens, self.heads, self.head_dim = n_pages, page_tokens, heads, head_dim
        self.struct = CacheStruct(data.data_ptr(), n_pages, data.stride(0), data.stride(1), page_tokens, heads, head_dim, TYPES[dtype])
        self.address = C.addressof(self.struct)


def qsgd_cache_write(cache, table, lengths, k, v, status_dev, starts=None, stream=None):
    """Quantises k and v, [rows, heads, head_dim], into the cache: the last tokens of every sequence (one each, or rows
    starts[b] to starts[b + 1]). table [sequences, pages], lengths (these tokens included) and starts are int32."""
    _check(_native.cache_store(True, cache.address, cache.data, table, lengths, starts, k, v, status_dev, stream))


def qsgd_cache_read(cache, table, lengths, k, v, status_dev, starts=None, stream=None):
    """Reads the last tokens of every sequence back into k and v; arguments as qsgd_cache_write."""
    _check(_native.cache_store(False, cache.address, cache.data, table, lengths, starts, k, v, status_dev, stream))


def qsgd_cache_attend_workspace_bytes(cache, q_heads):
    return int(lib().qsgd_cache_attend_workspace_bytes(C.byref(cache.struct), q_heads))


def qsgd_cache_attend(cache, table, lengths, q, out, workspace, status_dev, starts=None, scale=None, lse=None, stream=None):
    """out <- attention of q, [rows, q_heads, head_dim], over the cache: a row sees the tokens up to its own. scale defaults
    to 1 / sqrt(head_dim); lse, [rows, q_heads] in fp32, receives the logarithm of the sum of exponentials."""
    _check(_native.cache_attend(cache.address, cache.data, table, lengths, starts, q, out, workspace, status_dev, scale, lse, stream))


def qsgd_quantize_rows(x, codes, scale, stream=None):
    """Rows of x (fp32, fp16 or bf16) as int8 codes and an fp32 scale each."""
    _check(_native.quantize_rows(x, codes, scale, stream))


def qsgd_matmul_i8(a, a_scale, b, b_scale, out, bias=None, stream=None, status_dev=None):
    """out <- (a b^T) * a_scale[:, None] * b_scale + bias, for int8 a and b; the sum is exact."""
    _check(_native.matmul_i8(a, a_scale, b, b_scale, out, bias, status_dev, stream))


def qsgd_linear_i8_workspace_bytes(rows, cols):
    return int(lib().qsgd_linear_i8_workspace_bytes(rows, cols))


def qsgd_linear_i8(x, w, w_scale, out, workspace, bias=None, stream=None, status_dev=None):
    """out <- x w^T + bias with the rows of x quantised on the way; w and w_scale as qsgd_quantize_rows leaves them."""
    _check(_native.linear_i8(x, w, w_scale, out, workspace, bias, status_dev, stream))


def quantize_rows_alloc(x, stream=None):
    """Allocates codes whose rows begin on 16-byte boundaries (what the products read fastest) and scales, then calls
    qsgd_quantize_rows. Returns (codes, scale)."""
    rows, cols = x.shape
    codes = torch.zeros(rows, (cols + 15) // 16 * 16, dtype=torch.int8, device=x.device)[:, :cols]
    scale = torch.empty(rows, dtype=torch.float32, device=x.device)
    qsgd_quantize_rows(x, codes, scale, stream)
    return codes, scale


# ------------------------------- conveniences (allocation only) -----------------------------
def new_status(device="cuda"):
    return torch.zeros(1, dtype=torch.int32, device=device)


def encode_alloc(g, bucket, s, norm_kind, code_kind, seed, step, worker, capacity=None,
                 stream=None):
    """Allocates the message, info words, workspace and status, then calls qsgd_encode.
    Returns (out, out_bits, status_dev); synchronise before reading them on the host."""
    n = g.numel()
    cap = qsgd_message_capacity(n, bucket, s, code_kind) if capacity is None else capacity
    out = torch.empty(cap, dtype=torch.uint8, device=g.device)
    out_bits = torch.zeros(4, dtype=torch.int64, device=g.device)
    wsb = qsgd_workspace_bytes(n, bucket, s, code_kind)
    ws = torch.empty(max(wsb, 16), dtype=torch.uint8, device=g.device)
    status = new_status(g.device)
    qsgd_encode(g, bucket, s, norm_kind, code_kind, seed, step, worker, out, out_bits, ws, status,
                stream)
    return out, out_bits, status
