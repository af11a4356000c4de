"""ctypes binding for ``libdynaresize.so``: structures and functions named as in ``dynaresize.h``."""
from __future__ import annotations

import ctypes as C
import os

_DIR = os.path.dirname(os.path.abspath(__file__))
lib_path = os.path.join(_DIR, "libdynaresize.so")

DR_OK = 0
DR_ERR_INVALID, DR_ERR_UNSUPPORTED, DR_ERR_SIZE, DR_ERR_ALIGN, DR_ERR_NOMEM = -1, -2, -3, -4, -5
DR_ERR_CUDA, DR_ERR_BUDGET, DR_ERR_SINK, DR_ERR_TIMEOUT, DR_ERR_STATE = -6, -7, -8, -9, -10
DR_VERSION = 1
DR_SRC_FSDP_FLAT = 1
DR_DST_ROLLOUT_FUSED = 1
DR_F32, DR_BF16, DR_FP8_E4M3_B128 = 1, 2, 3
DR_MAX_STAGE_BUFS = 8
DR_STAGE_HOST_OFFSETS = 1
DR_STAGE_UNORDERED = 2
DR_STREAM_UNORDERED = 1
DR_STAGE_DIR_OUT, DR_STAGE_DIR_IN = 0, 1

EXPORTS = ["dr_plan_create", "dr_plan_create_host", "dr_plan_window_host", "dr_plan_query", "dr_plan_tensor", "dr_plan_segment",
           "dr_reshard", "dr_reshard_inverse", "dr_plan_group", "dr_reshard_groups", "dr_reshard_static", "dr_plan_ranges", "dr_reshard_push", "dr_reshard_stream", "dr_shard_range", "dr_stage_out", "dr_stage_in", "dr_stage_begin", "dr_stage_wait_buffer", "dr_stage_poll", "dr_stage_end", "dr_plan_destroy", "dr_strerror",
           "dr_last_error", "dr_probe_stream", "dr_host_copy", "dr_diag_bulk_wait_failures", "dr_diag_bulk_starve", "dr_ctl_create", "dr_ctl_observe", "dr_ctl_break_even", "dr_ctl_destroy",
           "dr_quant_rows", "dr_linear_create", "dr_linear_destroy", "dr_linear_forward", "dr_linear_dgrad", "dr_linear_wgrad", "dr_diag_linear_wait_failures", "dr_diag_linear_waits"]

u8, u32, u64, i64, vp = C.c_uint8, C.c_uint32, C.c_uint64, C.c_int64, C.c_void_p


class dr_model_spec(C.Structure):
    _fields_ = [("struct_size", u32), ("version", u32), ("n_layers", u32), ("hidden", u32), ("n_q_heads", u32),
                ("n_kv_heads", u32), ("head_dim", u32), ("ffn", u32), ("vocab", u32), ("n_experts", u32),
                ("moe_ffn", u32), ("tied_embeddings", u8), ("qk_norm", u8), ("pad", u8 * 2)]


class dr_src_layout(C.Structure):
    _fields_ = [("struct_size", u32), ("kind", u32), ("dtype", u32), ("world", u32), ("rank", u32),
                ("gathered", u32), ("align_elems", u32)]


class dr_dst_layout(C.Structure):
    _fields_ = [("struct_size", u32), ("kind", u32), ("dtype", u32), ("moe_tp", u32), ("arena_align_bytes", u32),
                ("kv_replicate", u32), ("vocab_pad", u32), ("moe_ep", u32), ("moe_ep_rank", u32)]


class dr_plan_info(C.Structure):
    _fields_ = [(n, u64) for n in ("flat_elems", "shard_elems", "src_bytes", "dst_bytes", "n_tensors", "n_segments",
                                   "n_tiles", "elems_moved", "bytes_moved_fwd", "bytes_moved_inv",
                                   "quant_elems", "quant_blocks", "n_groups", "bulk_forward")]


class dr_group_desc(C.Structure):
    _fields_ = [("first_tensor", u32), ("n_tensors", u32), ("elems", u64), ("bytes_moved", u64)]


class dr_range(C.Structure):
    _fields_ = [("off", u64), ("bytes", u64)]


class dr_tensor_desc(C.Structure):
    _fields_ = [("name", C.c_char * 64), ("arena_off", u64), ("rows", u64), ("cols", u64), ("alias_of", i64),
                ("elem_size", u32), ("quantised", u32), ("scale_off", u64), ("scale_rows", u64), ("scale_cols", u64)]


class dr_segment_desc(C.Structure):
    _fields_ = [("dst_off", u64), ("src_off", u64), ("rows", u64), ("row_len", u64), ("src_row_stride", u64),
                ("dst_row_stride", u64), ("vector_bytes", u32), ("tensor", u32)]


dr_chunk_fn = C.CFUNCTYPE(C.c_int, vp, u64, u64, vp, u64)


class dr_stage_desc(C.Structure):
    _fields_ = [("struct_size", u32), ("n_bufs", u32), ("dev_ptr", vp * 8), ("bytes", u64 * 8), ("order", u32 * 8),
                ("budget_bytes", u64), ("chunk_bytes", u64), ("host_arena", vp), ("host_arena_bytes", u64),
                ("callback", dr_chunk_fn), ("user", vp), ("relay_dev", vp * 8), ("first_chunk", u64),
                ("wait_event", vp), ("ready_events", vp * 8), ("timeout_ms", u32), ("flags", u32),
                ("host_offset", u64 * 8), ("caller_stream", vp), ("done_event", vp)]


class dr_stage_stats(C.Structure):
    _fields_ = [("bytes", u64), ("chunks_done", u64), ("n_chunks", u64), ("elapsed_ms", C.c_double),
                ("link_gbs", C.c_double), ("pinned_high_water_bytes", u64), ("ready_ms", C.c_double * 8)]


class dr_stream_desc(C.Structure):
    _fields_ = [("struct_size", u32), ("flags", u32), ("host_src", vp), ("host_src_bytes", u64), ("dst_dev", vp),
                ("dst_bytes", u64), ("host_dst", vp), ("host_dst_bytes", u64), ("window_dev", vp), ("window_bytes", u64),
                ("chunk_bytes", u64), ("timeout_ms", u32), ("pad", u32), ("caller_stream", vp), ("wait_event", vp),
                ("done_event", vp)]


class dr_stream_stats(C.Structure):
    _fields_ = [("h2d_bytes", u64), ("d2h_bytes", u64), ("n_chunks", u64), ("kernels", u64), ("elapsed_ms", C.c_double)]


class dr_ctl_config(C.Structure):
    _fields_ = [("struct_size", u32), ("n_topologies", u32), ("initial", u32), ("consecutive", u32), ("dwell_steps", u32),
                ("cooldown_steps", u32), ("enter_threshold", C.c_double), ("exit_threshold", C.c_double)]


class dr_linear_desc(C.Structure):
    _fields_ = [("struct_size", u32), ("dtype", u32), ("n_groups", u32), ("pad", u32), ("out_features", u64),
                ("in_features", u64), ("weight_dev", vp), ("weight_bytes", u64), ("weight_ld", u64), ("scale_dev", vp),
                ("scale_bytes", u64), ("scale_ld", u64)]


class DrError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {dr_strerror(status)} ({status}): {dr_last_error()}")


_lib = None


def lib() -> C.CDLL:
    """The loaded C-ABI library.  Raises if it has not been built: there is no other code path."""
    global _lib
    if _lib is None:
        if not os.path.exists(lib_path):
            raise ImportError(f"{lib_path} is missing: run `python -m paper_2607_22614_b200.build` "
                              "(the CUDA library is the only implementation)")
        L = C.CDLL(lib_path)
        P = C.POINTER
        L.dr_plan_create.argtypes = [P(dr_model_spec), P(dr_src_layout), P(dr_dst_layout), u32, u32, P(vp)]
        L.dr_plan_create_host.argtypes = L.dr_plan_create.argtypes
        L.dr_plan_window_host.argtypes = [vp, u64, u64, P(vp)]
        L.dr_plan_query.argtypes = [vp, P(dr_plan_info)]
        L.dr_plan_tensor.argtypes = [vp, u32, P(dr_tensor_desc)]
        L.dr_plan_segment.argtypes = [vp, u64, P(dr_segment_desc)]
        L.dr_reshard.argtypes = [vp, vp, u64, vp, u64, vp]
        L.dr_reshard_inverse.argtypes = [vp, vp, u64, vp, u64, vp]
        L.dr_reshard_static.argtypes = [vp, vp, u64, vp, u64, vp]
        L.dr_plan_ranges.argtypes = [vp, u64, P(dr_range), P(u64)]
        L.dr_reshard_push.argtypes = [vp, vp, u64, P(vp), u32, u64, vp]
        L.dr_plan_group.argtypes = [vp, u32, P(dr_group_desc)]
        L.dr_reshard_groups.argtypes = [vp, u32, u32, vp, u64, vp, u64, vp]
        L.dr_stage_out.argtypes = [vp, P(dr_stage_desc), P(dr_stage_stats)]
        L.dr_stage_in.argtypes = [vp, P(dr_stage_desc), P(dr_stage_stats)]
        L.dr_stage_begin.argtypes = [vp, P(dr_stage_desc), C.c_int, P(vp)]
        L.dr_stage_wait_buffer.argtypes = [vp, u32, u32]
        L.dr_stage_poll.argtypes = [vp, P(C.c_int)]
        L.dr_stage_end.argtypes = [vp, P(dr_stage_stats)]
        L.dr_reshard_stream.argtypes = [vp, P(dr_stream_desc), P(dr_stream_stats)]
        L.dr_plan_destroy.argtypes = [vp]
        L.dr_shard_range.argtypes = [u64, u32, u32, P(u64), P(u64), P(u64)]
        L.dr_probe_stream.argtypes = [u32, vp, vp, u64, vp]
        L.dr_host_copy.argtypes = [vp, vp, u64, u32]
        L.dr_diag_bulk_wait_failures.argtypes = [P(u64)]
        L.dr_diag_bulk_starve.argtypes = [C.c_int]
        L.dr_ctl_create.argtypes = [P(dr_ctl_config), P(vp)]
        L.dr_ctl_observe.argtypes = [vp, C.c_double, C.c_double, P(C.c_int32), P(u32)]
        L.dr_ctl_break_even.argtypes = [C.c_double, C.c_double, C.c_double, P(C.c_double)]
        L.dr_ctl_destroy.argtypes = [vp]
        L.dr_quant_rows.argtypes = [vp, u32, u64, u64, vp, u32, u64, u64, vp, u64, vp, u64, vp]
        L.dr_linear_create.argtypes = [P(dr_linear_desc), P(vp)]
        L.dr_linear_destroy.argtypes = [vp]
        L.dr_linear_forward.argtypes = [vp, vp, u64, vp, u64, u64, vp, vp, u64, u32, vp]
        L.dr_linear_dgrad.argtypes = [vp, vp, u64, u64, vp, vp, u64, u32, vp]
        L.dr_linear_wgrad.argtypes = [vp, vp, u64, vp, u64, u64, vp, vp, u64, u32, vp]
        L.dr_diag_linear_wait_failures.argtypes = [P(u64)]
        L.dr_diag_linear_waits.argtypes = [u32, u32]
        for n in EXPORTS:
            getattr(L, n).restype = C.c_int
        L.dr_strerror.argtypes = [C.c_int]
        L.dr_strerror.restype = C.c_char_p
        L.dr_last_error.argtypes = []
        L.dr_last_error.restype = C.c_char_p
        _lib = L
    return _lib


# ---- struct helpers ----------------------------------------------------------------------------
def model_spec(spec: dict) -> dr_model_spec:
    return dr_model_spec(struct_size=C.sizeof(dr_model_spec), version=DR_VERSION, n_layers=spec["n_layers"],
                         hidden=spec["hidden"], n_q_heads=spec["n_q_heads"], n_kv_heads=spec["n_kv_heads"],
                         head_dim=spec["head_dim"], ffn=spec.get("ffn", 0), vocab=spec["vocab"],
                         n_experts=spec.get("n_experts", 0), moe_ffn=spec.get("moe_ffn", 0),
                         tied_embeddings=int(spec.get("tied", 0)), qk_norm=int(spec.get("qk_norm", 1)))


def src_layout(world=1, rank=0, gathered=True, align_elems=1) -> dr_src_layout:
    return dr_src_layout(struct_size=C.sizeof(dr_src_layout), kind=DR_SRC_FSDP_FLAT, dtype=DR_F32, world=world,
                         rank=rank, gathered=int(gathered), align_elems=align_elems)


def dst_layout(dtype=DR_BF16, arena_align_bytes=256, moe_tp=1, kv_replicate=False, vocab_pad=0, moe_ep=1,
               moe_ep_rank=0) -> dr_dst_layout:
    return dr_dst_layout(struct_size=C.sizeof(dr_dst_layout), kind=DR_DST_ROLLOUT_FUSED, dtype=dtype, moe_tp=moe_tp,
                         arena_align_bytes=arena_align_bytes, kv_replicate=int(kv_replicate), vocab_pad=vocab_pad,
                         moe_ep=moe_ep, moe_ep_rank=moe_ep_rank)


def _current_stream(stream):
    """cudaStream_t of `stream` (a torch stream, a raw handle, or None = torch's current stream)."""
    if stream is None:
        import torch
        # without a CUDA device the descriptor can still be built (argument checks); NULL = legacy default stream
        if torch.cuda.is_initialized() or torch.cuda.is_available():
            return torch.cuda.current_stream().cuda_stream
        return None
    return getattr(stream, "cuda_stream", stream)


def stage_desc(dev_ptrs, sizes, budget, chunk=0, order=None, host_arena=None, host_arena_bytes=0, callback=None,
               relay_dev=None, first_chunk=0, wait_event=None, ready_events=None, timeout_ms=0,
               host_offsets=None, caller_stream=None, done_event=None, unordered=False) -> dr_stage_desc:
    """Fill a dr_stage_desc.  caller_stream=None names torch's current stream: the call's first copy then waits
    for whatever has been enqueued there (the fills or kernels that produced the device buffers)."""
    d = dr_stage_desc()
    d.struct_size = C.sizeof(dr_stage_desc)
    d.n_bufs = len(dev_ptrs)
    for i, (p, n) in enumerate(zip(dev_ptrs, sizes)):
        d.dev_ptr[i] = p
        d.bytes[i] = n
    for i, o in enumerate(order if order is not None else range(len(dev_ptrs))):
        d.order[i] = o
    d.budget_bytes, d.chunk_bytes, d.first_chunk, d.timeout_ms = budget, chunk, first_chunk, timeout_ms
    d.host_arena, d.host_arena_bytes = host_arena, host_arena_bytes
    if callback is not None:
        d.callback = callback
    for i, p in enumerate(relay_dev or []):
        d.relay_dev[i] = p
    d.wait_event = wait_event
    for i, e in enumerate(ready_events or []):
        d.ready_events[i] = e
    if host_offsets is not None:
        d.flags |= DR_STAGE_HOST_OFFSETS
        for i, o in enumerate(host_offsets):
            d.host_offset[i] = o
    if unordered:
        d.flags |= DR_STAGE_UNORDERED
    else:
        d.caller_stream = _current_stream(caller_stream)
    d.done_event = done_event
    return d


# ---- the C calls, same names, status codes returned as-is ---------------------------------------
def dr_plan_create(spec, src, dst, tp, rank):
    h = vp()
    rc = lib().dr_plan_create(C.byref(spec), C.byref(src), C.byref(dst), tp, rank, C.byref(h))
    return rc, h


def dr_plan_create_host(spec, src, dst, tp, rank):
    h = vp()
    rc = lib().dr_plan_create_host(C.byref(spec), C.byref(src), C.byref(dst), tp, rank, C.byref(h))
    return rc, h


def dr_plan_window_host(plan, src_elem_lo, src_elem_hi):
    h = vp()
    return lib().dr_plan_window_host(plan, src_elem_lo, src_elem_hi, C.byref(h)), h


def dr_plan_query(plan):
    info = dr_plan_info()
    return lib().dr_plan_query(plan, C.byref(info)), info


def dr_plan_tensor(plan, i):
    t = dr_tensor_desc()
    return lib().dr_plan_tensor(plan, i, C.byref(t)), t


def dr_plan_segment(plan, i):
    s = dr_segment_desc()
    return lib().dr_plan_segment(plan, i, C.byref(s)), s


def dr_reshard(plan, src_dev, src_bytes, dst_dev, dst_bytes, cuda_stream):
    return lib().dr_reshard(plan, src_dev, src_bytes, dst_dev, dst_bytes, cuda_stream)


def dr_reshard_inverse(plan, rollout_dev, rollout_bytes, flat_dev, flat_bytes, cuda_stream):
    return lib().dr_reshard_inverse(plan, rollout_dev, rollout_bytes, flat_dev, flat_bytes, cuda_stream)


def dr_plan_group(plan, g):
    d = dr_group_desc()
    return lib().dr_plan_group(plan, g, C.byref(d)), d


def dr_reshard_groups(plan, first, count, src_dev, src_bytes, dst_dev, dst_bytes, cuda_stream):
    return lib().dr_reshard_groups(plan, first, count, src_dev, src_bytes, dst_dev, dst_bytes, cuda_stream)


def dr_plan_ranges(plan):
    """(status, [(off, bytes), ...]): the coalesced arena byte ranges the plan's repack writes."""
    n = u64()
    rc = lib().dr_plan_ranges(plan, 0, None, C.byref(n))
    if rc:
        return rc, []
    arr = (dr_range * max(n.value, 1))()
    rc = lib().dr_plan_ranges(plan, n.value, arr, C.byref(n))
    return rc, [(arr[i].off, arr[i].bytes) for i in range(n.value)]


def dr_reshard_push(plan, src_dev, src_bytes, dst_devs, dst_bytes, cuda_stream):
    arr = (vp * len(dst_devs))(*dst_devs)
    return lib().dr_reshard_push(plan, src_dev, src_bytes, arr, len(dst_devs), dst_bytes, cuda_stream)


def dr_reshard_static(plan, src_dev, src_bytes, dst_dev, dst_bytes, cuda_stream):
    """dr_reshard without any device allocation: the segment table goes into the library's fixed
    1 MiB table (at most 16 384 segments).  For workers whose memory pool owns the whole GPU, or whose
    switch must not be stalled by the device synchronisation that cudaMalloc / cudaFree imply."""
    return lib().dr_reshard_static(plan, src_dev, src_bytes, dst_dev, dst_bytes, cuda_stream)


def dr_stage_out(plan, desc):
    st = dr_stage_stats()
    return lib().dr_stage_out(plan, C.byref(desc), C.byref(st)), st


def dr_stage_in(plan, desc):
    st = dr_stage_stats()
    return lib().dr_stage_in(plan, C.byref(desc), C.byref(st)), st


def dr_stage_begin(plan, desc, direction):
    """Starts dr_stage_out / dr_stage_in on a thread of the library's own; returns (status, job handle)."""
    job = vp()
    return lib().dr_stage_begin(plan, C.byref(desc), direction, C.byref(job)), job


def dr_stage_wait_buffer(job, buffer, timeout_ms=0):
    return lib().dr_stage_wait_buffer(job, buffer, timeout_ms)


def dr_stage_poll(job):
    done = C.c_int(0)
    return lib().dr_stage_poll(job, C.byref(done)), bool(done.value)


def dr_stage_end(job):
    st = dr_stage_stats()
    return lib().dr_stage_end(job, C.byref(st)), st


def stream_desc(host_src, host_src_bytes, dst_dev, dst_bytes, window_dev, window_bytes, chunk_bytes=0, host_dst=None,
                host_dst_bytes=0, timeout_ms=0, caller_stream=None, wait_event=None, done_event=None,
                unordered=False) -> dr_stream_desc:
    """Fill a dr_stream_desc; caller_stream=None names torch's current stream (see stage_desc)."""
    return dr_stream_desc(struct_size=C.sizeof(dr_stream_desc), flags=DR_STREAM_UNORDERED if unordered else 0,
                          host_src=host_src, host_src_bytes=host_src_bytes,
                          dst_dev=dst_dev, dst_bytes=dst_bytes, host_dst=host_dst, host_dst_bytes=host_dst_bytes,
                          window_dev=window_dev, window_bytes=window_bytes, chunk_bytes=chunk_bytes, timeout_ms=timeout_ms,
                          caller_stream=None if unordered else _current_stream(caller_stream), wait_event=wait_event,
                          done_event=done_event)


def dr_reshard_stream(plan, desc):
    st = dr_stream_stats()
    return lib().dr_reshard_stream(plan, C.byref(desc), C.byref(st)), st


DR_PROBE_READ, DR_PROBE_WRITE, DR_PROBE_COPY, DR_PROBE_NARROW, DR_PROBE_WIDEN, DR_PROBE_NARROW4, DR_PROBE_WIDEN4 = range(7)


def dr_probe_stream(mode, a_dev, b_dev, n_bytes, cuda_stream):
    return lib().dr_probe_stream(mode, a_dev, b_dev, n_bytes, cuda_stream)


def dr_diag_bulk_wait_failures():
    n = u64()
    return lib().dr_diag_bulk_wait_failures(C.byref(n)), n.value


def dr_diag_linear_wait_failures():
    n = u64()
    return lib().dr_diag_linear_wait_failures(C.byref(n)), n.value


def dr_diag_linear_waits(limit_us, starve):
    return lib().dr_diag_linear_waits(limit_us, starve)


def dr_diag_bulk_starve(on):
    return lib().dr_diag_bulk_starve(int(on))


def dr_host_copy(dst_host, src_host, n_bytes, threads=0):
    return lib().dr_host_copy(dst_host, src_host, n_bytes, threads)


def dr_shard_range(flat_elems, world, rank):
    b, e, s = u64(), u64(), u64()
    rc = lib().dr_shard_range(flat_elems, world, rank, C.byref(b), C.byref(e), C.byref(s))
    return rc, b.value, e.value, s.value


def dr_ctl_create(n_topologies, initial=0, enter=0.2, exit=0.1, consecutive=3, dwell=5, cooldown=11):
    cfg = dr_ctl_config(struct_size=C.sizeof(dr_ctl_config), n_topologies=n_topologies, initial=initial,
                        consecutive=consecutive, dwell_steps=dwell, cooldown_steps=cooldown, enter_threshold=enter,
                        exit_threshold=exit)
    h = vp()
    return lib().dr_ctl_create(C.byref(cfg), C.byref(h)), h


def dr_ctl_observe(ctl, t_rollout, t_train):
    move, topo = C.c_int32(), u32()
    rc = lib().dr_ctl_observe(ctl, t_rollout, t_train, C.byref(move), C.byref(topo))
    return rc, move.value, topo.value


def dr_ctl_break_even(resize_cost_s, step_before_s, step_after_s):
    out = C.c_double()
    return lib().dr_ctl_break_even(resize_cost_s, step_before_s, step_after_s, C.byref(out)), out.value


def dr_ctl_destroy(ctl):
    return lib().dr_ctl_destroy(ctl)


DR_ROWS_PLAIN, DR_ROWS_SWIGLU = 0, 1


def dr_quant_rows(x_dev, x_dtype, ldx, src_rows, row_index_dev, form, rows, cols, codes_dev, ld_codes, scales_dev, ld_scales,
                  cuda_stream):
    return lib().dr_quant_rows(x_dev, x_dtype, ldx, src_rows, row_index_dev, form, rows, cols, codes_dev, ld_codes,
                               scales_dev, ld_scales, cuda_stream)


def dr_linear_create(desc):
    h = vp()
    return lib().dr_linear_create(C.byref(desc), C.byref(h)), h


def dr_linear_destroy(lin):
    return lib().dr_linear_destroy(lin)


def dr_linear_forward(lin, x_dev, ldx, x_scale_dev, ld_scale, rows, offsets_dev, y_dev, ldy, y_dtype, cuda_stream):
    return lib().dr_linear_forward(lin, x_dev, ldx, x_scale_dev, ld_scale, rows, offsets_dev, y_dev, ldy, y_dtype, cuda_stream)


def dr_linear_dgrad(lin, dy_dev, lddy, rows, offsets_dev, dx_dev, lddx, dx_dtype, cuda_stream):
    return lib().dr_linear_dgrad(lin, dy_dev, lddy, rows, offsets_dev, dx_dev, lddx, dx_dtype, cuda_stream)


def dr_linear_wgrad(lin, x_dev, ldx, dy_dev, lddy, rows, offsets_dev, dw_dev, lddw, accumulate, cuda_stream):
    return lib().dr_linear_wgrad(lin, x_dev, ldx, dy_dev, lddy, rows, offsets_dev, dw_dev, lddw, accumulate, cuda_stream)


def dr_plan_destroy(plan):
    return lib().dr_plan_destroy(plan)


def dr_strerror(status: int) -> str:
    return lib().dr_strerror(status).decode()


def dr_last_error() -> str:
    return lib().dr_last_error().decode()


# ---- convenience wrapper (raises instead of returning codes; still marshalling only) -------------
class StageJob:
    """A deferred stage call (dr_stage_begin): poll() tells whether the pump has returned, end() collects it."""

    def __init__(self, handle, desc):
        self.handle, self.desc = handle, desc

    def poll(self) -> bool:
        rc, done = dr_stage_poll(self.handle)
        if rc:
            raise DrError(rc, "dr_stage_poll")
        return done

    def wait_buffer(self, buffer: int, timeout_ms: int = 0) -> None:
        """Blocks until buffer `buffer` of a stage-in job is resident (dr_stage_wait_buffer)."""
        rc = dr_stage_wait_buffer(self.handle, buffer, timeout_ms)
        if rc:
            raise DrError(rc, "dr_stage_wait_buffer")

    def end(self):
        if self.handle is None:
            raise RuntimeError("job already ended")
        rc, st = dr_stage_end(self.handle)
        self.handle = None
        if rc:
            e = DrError(rc, "dr_stage_end")
            e.stats = st
            raise e
        return st


class Plan:
    """Owns one ``dr_plan``.  ``host_only=True`` builds the planner's tables without touching CUDA."""

    def __init__(self, spec: dict, *, world=1, rank=0, gathered=True, align_elems=1, tp=1, tp_rank=0,
                 dtype=DR_BF16, arena_align_bytes=256, host_only=False, moe_tp=1, kv_replicate=False, vocab_pad=0,
                 moe_ep=1, moe_ep_rank=0):
        create = dr_plan_create_host if host_only else dr_plan_create
        rc, self.handle = create(model_spec(spec), src_layout(world, rank, gathered, align_elems),
                                 dst_layout(dtype, arena_align_bytes, moe_tp, kv_replicate, vocab_pad, moe_ep,
                                            moe_ep_rank), tp, tp_rank)
        if rc:
            self.handle = None
            raise DrError(rc, "dr_plan_create")
        rc, self.info = dr_plan_query(self.handle)
        if rc:
            raise DrError(rc, "dr_plan_query")
        self.experts = spec.get("n_experts", 0) // max(1, moe_ep)  # held by this rank

    def window(self, src_elem_lo, src_elem_hi):
        """Host-only plan for the source window [lo, hi) (what one chunk of the streamed repack covers)."""
        rc, h = dr_plan_window_host(self.handle, src_elem_lo, src_elem_hi)
        if rc:
            raise DrError(rc, "dr_plan_window_host")
        w = Plan.__new__(Plan)
        w.handle = h
        w.experts = self.experts
        rc, w.info = dr_plan_query(h)
        return w

    def close(self):
        if getattr(self, "handle", None):
            dr_plan_destroy(self.handle)
            self.handle = None

    __del__ = close

    def tensors(self):
        out = []
        for i in range(self.info.n_tensors):
            rc, t = dr_plan_tensor(self.handle, i)
            if rc:
                raise DrError(rc, "dr_plan_tensor")
            out.append(t)
        return out

    def segments(self):
        out = []
        for i in range(self.info.n_segments):
            rc, s = dr_plan_segment(self.handle, i)
            if rc:
                raise DrError(rc, "dr_plan_segment")
            out.append(s)
        return out

    _stream = staticmethod(_current_stream)

    def view(self, arena, name):
        """Rollout tensor `name` ("layers.0.qkv", "layers.3.w13", ...) of `arena` (a uint8 CUDA tensor that dr_reshard writes), as
        (payload [rows, cols] in its own type, block scales or None)."""
        import torch
        t = next((t for t in self.tensors() if t.name.decode() == name), None)
        if t is None:
            raise KeyError(f"the plan has no rollout tensor {name!r}")

        def part(off, rows, cols, dtype, size):
            return arena[off:off + rows * cols * size].view(dtype).view(rows, cols)

        types = {1: torch.float8_e4m3fn, 2: torch.bfloat16, 4: torch.float32}
        return (part(t.arena_off, t.rows, t.cols, types[t.elem_size], t.elem_size),
                part(t.scale_off, t.scale_rows, t.scale_cols, torch.float32, 4) if t.quantised else None)

    def linear(self, arena, name, n_groups=None):
        """The Linear layer over rollout tensor `name` of `arena`.  n_groups: experts stacked in w13 / w2; taken from the plan
        when it is None."""
        weight, scale = self.view(arena, name)
        if weight.element_size() == 4:
            raise TypeError("a linear layer needs bf16 or fp8 weights")
        if n_groups is None:
            n_groups = max(1, self.experts) if name.rsplit(".", 1)[-1] in ("w13", "w2") else 1
        return Linear(weight, scale, n_groups=n_groups)

    def reshard(self, src, dst, stream=None):
        """src: CUDA tensor holding the flat fp32 buffer; dst: CUDA tensor holding the rollout arena."""
        rc = dr_reshard(self.handle, src.data_ptr(), src.numel() * src.element_size(), dst.data_ptr(),
                        dst.numel() * dst.element_size(), self._stream(stream))
        if rc:
            raise DrError(rc, "dr_reshard")

    def ranges(self):
        rc, out = dr_plan_ranges(self.handle)
        if rc:
            raise DrError(rc, "dr_plan_ranges")
        return out

    def reshard_push(self, src, dsts, stream=None):
        """Repack src and store the result into every arena of dsts (CUDA tensors, or raw device pointers with
        the plan's dst_bytes behind them)."""
        ptrs = [d.data_ptr() if hasattr(d, "data_ptr") else int(d) for d in dsts]
        nbytes = min([d.numel() * d.element_size() for d in dsts if hasattr(d, "numel")] or [self.info.dst_bytes])
        rc = dr_reshard_push(self.handle, src.data_ptr(), src.numel() * src.element_size(), ptrs, nbytes,
                             self._stream(stream))
        if rc:
            raise DrError(rc, "dr_reshard_push")

    def reshard_groups(self, first, count, src, dst, stream=None):
        """Repack only groups [first, first + count) (0: embed, l + 1: layer l, last: final norm and lm_head)."""
        rc = dr_reshard_groups(self.handle, first, count, src.data_ptr(), src.numel() * src.element_size(), dst.data_ptr(),
                               dst.numel() * dst.element_size(), self._stream(stream))
        if rc:
            raise DrError(rc, "dr_reshard_groups")

    def reshard_inverse(self, rollout, flat, stream=None):
        rc = dr_reshard_inverse(self.handle, rollout.data_ptr(), rollout.numel() * rollout.element_size(),
                                flat.data_ptr(), flat.numel() * flat.element_size(), self._stream(stream))
        if rc:
            raise DrError(rc, "dr_reshard_inverse")

    def reshard_stream(self, desc):
        rc, st = dr_reshard_stream(self.handle, desc)
        if rc:
            raise DrError(rc, "dr_reshard_stream")
        return st

    def stage_out(self, desc):
        rc, st = dr_stage_out(self.handle, desc)
        if rc:
            e = DrError(rc, "dr_stage_out")
            e.stats = st
            raise e
        return st

    def stage_in(self, desc):
        rc, st = dr_stage_in(self.handle, desc)
        if rc:
            e = DrError(rc, "dr_stage_in")
            e.stats = st
            raise e
        return st

    def stage_begin(self, desc, direction):
        """dr_stage_begin: the pump runs on the library's thread; returns a StageJob (keep `desc` and its buffers alive)."""
        rc, job = dr_stage_begin(self.handle, desc, direction)
        if rc:
            raise DrError(rc, "dr_stage_begin")
        return StageJob(job, desc)


def _elsewhere(t, what, device):
    """The error for an operand that does not live on GPU `device`: a kernel of one GPU must not get another's addresses."""
    return ValueError(f"{what} must be on GPU {device}, not on " + (f"GPU {t.get_device()}" if t.is_cuda else "the CPU"))


def _matrix(t, what, device):
    """(rows, columns, elements between rows) of a matrix with contiguous rows on GPU `device`."""
    if t.dim() != 2:
        raise ValueError(f"{what} must be a CUDA matrix")
    if t.get_device() != device:
        raise _elsewhere(t, what, device)
    rows, cols = t.shape
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{what} must have contiguous rows")
    return rows, cols, ld if rows > 1 else cols  # torch gives any stride to a matrix of one row


_codes = None  # torch dtype -> DR_BF16 / DR_F32


def _code_of(t, what):
    global _codes
    if _codes is None:
        import torch
        _codes = {torch.bfloat16: DR_BF16, torch.float32: DR_F32}
    code = _codes.get(t.dtype)
    if code is None:
        raise TypeError(f"{what} must be bfloat16 or float32, not {t.dtype}")
    return code


_code_types = None


def _holds_codes(t):
    """Whether t holds e4m3 codes: as torch's e4m3fn, or as bytes.  Other types of one byte (e5m2, e4m3fnuz, int8, bool) have other values."""
    global _code_types
    if _code_types is None:
        import torch
        _code_types = (torch.float8_e4m3fn, torch.uint8)
    return t.dtype in _code_types


_fns = {}


def _fn(name):
    """The C function itself, looked up once."""
    f = _fns.get(name)
    if f is None:
        f = _fns[name] = getattr(lib(), name)
    return f


def _current_device():
    """Index of the current GPU (from its second call on, torch's own accessor)."""
    global _current_device
    import torch
    _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return torch.cuda.current_device()


def _not_current(t, what):
    if not t.is_cuda:
        return ValueError(f"{what} must be a CUDA matrix")
    return ValueError(f"{what} is on GPU {t.get_device()}, which is not the current one: call under torch.cuda.device")


_raw_stream = None


def _stream_of(device, stream):
    """The handle of `stream`, or of the stream that is current on GPU `device` (torch's own accessor of the raw handle: building
    a Stream object for it takes 3 us, more than the launch)."""
    global _raw_stream
    if stream is not None:
        return getattr(stream, "cuda_stream", stream)
    if _raw_stream is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda index: torch.cuda.current_stream(index).cuda_stream)
    return _raw_stream(device)


def _refuse_autograd(what):
    """Raises while gradients are enabled: the kernels write through raw pointers, and the result would come back without a
    graph, as if nothing depended on `what`, which requires a gradient."""
    import torch
    if torch.is_grad_enabled():
        raise RuntimeError(f"{what} requires a gradient, which this call does not record: make it under torch.no_grad() or on detached "
                           "tensors, and take the gradients with Linear.dgrad and Linear.wgrad")


def _empty(rows, cols, dtype, device, stream):
    """An output of the call, from the memory of the stream that the call runs on: a block of the current stream's memory may
    still be used by work queued there, which `stream` does not wait for."""
    import torch
    if stream is None:
        return torch.empty(rows, cols, dtype=dtype, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(getattr(stream, "cuda_stream", stream), device=device)
    with torch.cuda.stream(stream):
        return torch.empty(rows, cols, dtype=dtype, device=device)


def quant_rows(x, codes=None, scales=None, *, row_index=None, swiglu=False, stream=None):
    """dr_quant_rows: x [source rows, cols] (2 * cols with swiglu: gate, then up; bf16 or fp32) -> (codes [rows, cols],
    scales [ceil(cols / 128), rows]).  row_index (int64) gathers rows.  Outputs that are not given are allocated.  All
    operands live on the current GPU.  `stream` (default: the current one) is where the call runs and where its allocated
    outputs belong; the caller orders the operands that other streams write, as with any torch call under that stream.  Not recorded by autograd (an x that requires a gradient is refused)."""
    device = x.get_device()
    if device < 0 or device != _current_device():
        raise _not_current(x, "x")
    src_rows, width, ldx = _matrix(x, "x", device)
    if x.requires_grad:
        _refuse_autograd("x")
    cols = width // 2 if swiglu else width
    if swiglu and width % 2:
        raise ValueError("x holds gate and up side by side: its column count must be even")
    rows, index = src_rows, None
    if row_index is not None:
        import torch
        if row_index.dtype != torch.int64 or row_index.dim() != 1 or not row_index.is_cuda or not row_index.is_contiguous():
            raise ValueError("row_index must be a contiguous int64 CUDA vector")
        if row_index.get_device() != device:
            raise _elsewhere(row_index, "row_index", device)
        rows, index = row_index.shape[0], row_index.data_ptr()
    blocks = -(-cols // 128)
    if codes is None or scales is None:
        import torch
        if codes is None:
            codes = _empty(rows, cols, torch.float8_e4m3fn, x.device, stream)
        if scales is None:
            scales = _empty(blocks, rows, torch.float32, x.device, stream)
    got_rows, got_cols, ld_codes = _matrix(codes, "codes", device)
    if got_rows != rows or got_cols != cols or not _holds_codes(codes):
        raise ValueError(f"codes must be {rows} x {cols} of float8_e4m3fn or uint8")
    got_blocks, got_rows, ld_scales = _matrix(scales, "scales", device)
    if got_rows != rows or got_blocks != blocks or _code_of(scales, "scales") != DR_F32:
        raise ValueError(f"scales must be fp32, {blocks} x {rows}")
    rc = _fn("dr_quant_rows")(x.data_ptr(), _code_of(x, "x"), ldx, src_rows, index, DR_ROWS_SWIGLU if swiglu else DR_ROWS_PLAIN,
                              rows, cols, codes.data_ptr(), ld_codes, scales.data_ptr(), ld_scales, _stream_of(device, stream))
    if rc:
        raise DrError(rc, "dr_quant_rows")
    return codes, scales


class Linear:
    """Owns one ``dr_linear``: a weight [n_groups * out, in] (bf16, or e4m3 codes with `scale`, one fp32 per 128 x 128
    block of the stacked matrix), its products and, for bf16, its gradients.  Keeps references to both tensors.  The weight
    and every operand of a product live on one GPU, which is the current one.  `stream` is as in quant_rows."""

    def __init__(self, weight, scale=None, n_groups=1):
        import torch
        self.device = weight.get_device()
        if self.device < 0 or self.device != _current_device():
            raise _not_current(weight, "weight")
        rows, cols, ld = _matrix(weight, "weight", self.device)
        fp8 = _holds_codes(weight)
        if not fp8 and weight.dtype != torch.bfloat16:
            raise TypeError(f"weight must be bfloat16 or e4m3 codes (float8_e4m3fn or uint8), not {weight.dtype}")
        if n_groups < 1 or rows % n_groups:
            raise ValueError("n_groups must divide the weight's rows")
        scale_rows = scale_cols = scale_ld = 0
        if scale is not None:
            scale_rows, scale_cols, scale_ld = _matrix(scale, "scale", self.device)
            if scale.dtype != torch.float32 or scale_rows != -(-rows // 128) or scale_cols != -(-cols // 128):
                raise ValueError("scale must be fp32 with one value for each 128 x 128 block of the weight")
        self.weight, self.scale, self.n_groups, self.fp8 = weight, scale, n_groups, fp8
        self.out_features, self.in_features = rows // n_groups, cols
        desc = dr_linear_desc(struct_size=C.sizeof(dr_linear_desc), dtype=DR_FP8_E4M3_B128 if fp8 else DR_BF16,
                              n_groups=n_groups, out_features=self.out_features, in_features=cols,
                              weight_dev=weight.data_ptr(), weight_bytes=((rows - 1) * ld + cols) * weight.element_size(), weight_ld=ld,
                              scale_dev=None if scale is None else scale.data_ptr(),
                              scale_bytes=4 * ((scale_rows - 1) * scale_ld + scale_cols) if scale is not None else 0,
                              scale_ld=scale_ld)
        rc, self.handle = dr_linear_create(desc)
        if rc:
            self.handle = None
            raise DrError(rc, "dr_linear_create")

    def close(self):
        if getattr(self, "handle", None):
            dr_linear_destroy(self.handle)
            self.handle = None

    def __del__(self):
        if lib is not None:  # at the interpreter's end the module may be gone before its objects
            self.close()

    def _operand(self, t, cols, what, fp8=False):
        rows, got, ld = _matrix(t, what, self.device)
        if got != cols:
            raise ValueError(f"{what} must have {cols} columns")
        if not _holds_codes(t) if fp8 else _code_of(t, what) != DR_BF16:
            raise TypeError(f"{what} has the wrong type: {t.dtype}")
        return rows, ld

    def _offsets(self, offsets):
        if offsets is None:
            return None
        import torch
        if offsets.dtype != torch.int32 or offsets.numel() != self.n_groups + 1 or not offsets.is_cuda or not offsets.is_contiguous():
            raise ValueError(f"offsets must be {self.n_groups + 1} int32 on the GPU")
        if offsets.get_device() != self.device:
            raise _elsewhere(offsets, "offsets", self.device)
        return offsets.data_ptr()

    def _out(self, out, rows, cols, dtype, like, stream):
        if out is None:
            import torch
            return _empty(rows, cols, dtype or torch.bfloat16, like.device, stream), cols
        got_rows, got_cols, ld = _matrix(out, "out", self.device)
        if got_rows != rows or got_cols != cols:
            raise ValueError(f"out must be {rows} x {cols}")
        return out, ld

    def forward(self, x, x_scale=None, offsets=None, out=None, out_dtype=None, stream=None):
        """dr_linear_forward: y = x W^T, for rows sorted by group where `offsets` (n_groups + 1, int32) is given.  An fp8
        layer takes quant_rows' codes and scales.  Rows of an allocated output that no group owns are not initialised.  Not
        recorded by autograd: operands that require a gradient are refused while gradients are enabled."""
        rows, ldx = self._operand(x, self.in_features, "x", self.fp8)
        if x.requires_grad or self.weight.requires_grad:
            _refuse_autograd("x or the weight")
        y, ldy = self._out(out, rows, self.out_features, out_dtype, x, stream)
        ps, lds = None, 0
        if x_scale is not None:
            blocks, cols, lds = _matrix(x_scale, "x_scale", self.device)
            if blocks != -(-self.in_features // 128) or cols < rows or _code_of(x_scale, "x_scale") != DR_F32:
                raise ValueError("x_scale must be fp32, one row for each block of 128 columns, one column for each row of x")
            ps = x_scale.data_ptr()
        rc = _fn("dr_linear_forward")(self.handle, x.data_ptr(), ldx, ps, lds, rows, self._offsets(offsets), y.data_ptr(), ldy,
                                      _code_of(y, "out"), _stream_of(self.device, stream))
        if rc:
            raise DrError(rc, "dr_linear_forward")
        return y

    __call__ = forward

    def dgrad(self, dy, offsets=None, out=None, out_dtype=None, stream=None):
        """dr_linear_dgrad: the gradient of x, dy W."""
        rows, lddy = self._operand(dy, self.out_features, "dy")
        dx, lddx = self._out(out, rows, self.in_features, out_dtype, dy, stream)
        rc = _fn("dr_linear_dgrad")(self.handle, dy.data_ptr(), lddy, rows, self._offsets(offsets), dx.data_ptr(), lddx,
                                    _code_of(dx, "out"), _stream_of(self.device, stream))
        if rc:
            raise DrError(rc, "dr_linear_dgrad")
        return dx

    def wgrad(self, x, dy, offsets=None, out=None, accumulate=False, stream=None):
        """dr_linear_wgrad: the gradient of the weight in fp32, dy^T x group by group; accumulate adds it to `out`."""
        rows, ldx = self._operand(x, self.in_features, "x")
        dy_rows, lddy = self._operand(dy, self.out_features, "dy")
        if rows != dy_rows:
            raise ValueError("x and dy must have the same rows")
        if accumulate and out is None:
            raise ValueError("accumulate adds to `out`: give one")
        import torch
        dw, lddw = self._out(out, self.n_groups * self.out_features, self.in_features, torch.float32, x, stream)
        if _code_of(dw, "out") != DR_F32:
            raise TypeError("the gradient of the weight is fp32")
        rc = _fn("dr_linear_wgrad")(self.handle, x.data_ptr(), ldx, dy.data_ptr(), lddy, rows, self._offsets(offsets),
                                    dw.data_ptr(), lddw, int(accumulate), _stream_of(self.device, stream))
        if rc:
            raise DrError(rc, "dr_linear_wgrad")
        return dw
