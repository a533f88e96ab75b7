"""Thin ctypes binding of libdblp.so: argument marshalling only, same names as include/dblp.h.

Device buffers are torch tensors (torch is used for device memory and streams, nothing else).  Every step of the path
runs in the library's kernels; if the library has not been built, loading fails with an error -- there is no fallback.
"""
import ctypes as C
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdblp.so")

DBLP_F32, DBLP_BF16, DBLP_F16 = 0, 1, 2
DBLP_LOSS_NONE, DBLP_LOSS_IID, DBLP_LOSS_GE, DBLP_LOSS_MICROBURST = 0, 1, 2, 3
DBLP_SUM, DBLP_MEAN, DBLP_OUT_BF16 = 0, 1, 2
DBLP_ACCUMULATE, DBLP_ATTENTION_CAUSAL, DBLP_ROTATE_INTERLEAVED = 1, 1, 2
ACTIVATIONS = {None: 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
DBLP_ORTHOGONALIZE_STEPS = 16
MUON_COEFFICIENTS = ((3.4445, -4.7750, 2.0315),) * 5        # a published choice: singular values to within about 0.7 .. 1.2
LOSS_KINDS = {"none": DBLP_LOSS_NONE, "iid": DBLP_LOSS_IID, "ge": DBLP_LOSS_GE, "microburst": DBLP_LOSS_MICROBURST}
HDR_BYTES = 32
COUNTER_FIELDS = ("n_arrived", "n_accepted", "n_dup", "n_stale", "n_invalid", "n_late")


class dblp_loss_model_t(C.Structure):
    _fields_ = [("kind", C.c_uint32), ("pad", C.c_uint32), ("t_drop", C.c_uint64), ("t_gb", C.c_uint64),
                ("t_bg", C.c_uint64), ("t_init_bad", C.c_uint64), ("t_drop_good", C.c_uint64),
                ("t_drop_bad", C.c_uint64), ("window_len", C.c_uint64), ("t_drop_in", C.c_uint64),
                ("t_drop_out", C.c_uint64)]


class dblp_counters_t(C.Structure):
    _fields_ = [("n_arrived", C.c_uint64), ("n_accepted", C.c_uint64), ("n_dup", C.c_uint64),
                ("n_stale", C.c_uint64), ("n_invalid", C.c_uint64), ("n_late", C.c_uint64), ("status", C.c_uint32),
                ("pad", C.c_uint32)]


class dblp_device_buffers_t(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("grads", "hdr_ring", "payload_ring", "delivered_bits", "arrival",
                                          "n_arrived", "recv_bitmap", "slot_key", "counters", "agg", "recv_cnt",
                                          "missing_cnt", "ok", "all_ok", "ws")] + [("ws_bytes", C.c_size_t),
                                                                                   ("sent_bits", C.c_void_p)]


MARK_FIELDS = ("begin", "packetize_end", "loss_begin", "loss_end", "receive_begin", "claim_end", "reduce_end",
               "bound_begin", "bound_end", "end")


class dblp_round_marks_t(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in MARK_FIELDS]


class dblp_heads_t(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class dblp_attention_t(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("batch", "q_tokens", "k_tokens", "q_heads", "kv_heads", "head_dim")] + [
        ("dtype", C.c_int), ("flags", C.c_uint32), ("scale", C.c_float), ("q_lens", C.c_void_p), ("k_lens", C.c_void_p)]


class dblp_norm_rotate_t(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("batch", "tokens", "q_heads", "k_heads", "head_dim", "rotary_dim")] + [
        ("dtype", C.c_int), ("weight_dtype", C.c_int), ("flags", C.c_uint32), ("eps", C.c_float), ("positions", C.c_void_p),
        ("position_stride", C.c_int64), ("freqs", C.c_void_p)]


class dblp_matrix_t(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("col_stride", C.c_int64)]


class dblp_linear_t(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("rows", "in_", "out")] + [
        (n, C.c_int) for n in ("dtype", "out_dtype", "bias_dtype", "activation")] + [("flags", C.c_uint32)]


class dblp_orthogonalize_t(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("batch", "rows", "cols")] + [("x_dtype", C.c_int), ("out_dtype", C.c_int),
                ("steps", C.c_uint32), ("coefficients", C.POINTER(C.c_float)), ("eps", C.c_float), ("scale", C.c_float)] + [
        (n, C.c_int64) for n in ("x_batch_stride", "x_row_stride", "out_batch_stride", "out_row_stride")]


class RoundMarks:
    """Timing events for the stages of a whole-round call (torch events; the library records them)."""

    def __init__(self):
        self.events = {n: torch.cuda.Event(enable_timing=True) for n in MARK_FIELDS}
        for e in self.events.values():
            e.record()                      # torch creates the CUDA event on first use; the library needs the handle
        self.struct = dblp_round_marks_t(**{n: e.cuda_event for n, e in self.events.items()})

    def ms(self, first, last):
        return self.events[first].elapsed_time(self.events[last])


class DblpError(RuntimeError):
    def __init__(self, status, what):
        super().__init__("%s: %s (%d): %s" % (what, lib().dblp_strerror(status).decode(), status,
                                              lib().dblp_last_error().decode()))
        self.status = status


_lib = None
EXPORTS = ("dblp_plan_create", "dblp_plan_destroy", "dblp_plan_query", "dblp_plan_tune_reduce", "dblp_plan_set_wire_format",
           "dblp_plan_set_shard",
           "dblp_workspace_bytes",
           "dblp_loss_model_from_rates", "dblp_packetize", "dblp_apply_loss", "dblp_apply_loss_static",
           "dblp_apply_loss_resend", "dblp_missing_bits", "dblp_stop_workspace_bytes", "dblp_aggregate_book_stop",
           "dblp_round_until_stop",
           "dblp_aggregate_book",
           "dblp_aggregate_claim", "dblp_aggregate_claim_grouped", "dblp_claim_workspace_bytes", "dblp_aggregate_bitmap", "dblp_aggregate_reduce", "dblp_aggregate_reduce_ex", "dblp_aggregate_reduce_atomic", "dblp_norm_scratch_count", "dblp_aggregate", "dblp_round_reset", "dblp_check_bound", "dblp_bound_ok", "dblp_clr",
           "dblp_select_bound", "dblp_round_send", "dblp_round_receive", "dblp_round_device", "dblp_round_host",
           "dblp_embed", "dblp_embed_grad_workspace_bytes", "dblp_embed_grad", "dblp_dropout", "dblp_dropout_grad",
           "dblp_attention_workspace_bytes", "dblp_attention", "dblp_attention_grad", "dblp_wait_timeouts",
           "dblp_norm_rotate", "dblp_norm_rotate_grad_workspace_bytes", "dblp_norm_rotate_grad",
           "dblp_linear_workspace_bytes", "dblp_linear", "dblp_linear_grad",
           "dblp_orthogonalize_workspace_bytes", "dblp_orthogonalize",
           "dblp_strerror", "dblp_last_error", "dblp_launch_count")


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libdblp.so is not built: run `python -m paper_2605_01989_b200.build` "
                              "(needs nvcc); there is no CPU fallback")
        L = C.CDLL(LIB_PATH)
        L.dblp_strerror.restype = C.c_char_p
        L.dblp_last_error.restype = C.c_char_p
        L.dblp_launch_count.restype = C.c_uint64
        L.dblp_select_bound.restype = C.c_uint32
        L.dblp_select_bound.argtypes = [C.c_double, C.c_double, C.c_double, C.c_uint32, C.c_uint32, C.c_int, C.c_int,
                                        C.c_uint32]
        L.dblp_clr.argtypes = [C.c_double, C.c_double, C.c_double]
        L.dblp_loss_model_from_rates.argtypes = [C.c_int, C.c_double, C.c_double, C.c_double, C.c_double, C.c_double,
                                                 C.c_uint64, C.POINTER(dblp_loss_model_t)]
        vp, i64, u64, u32 = C.c_void_p, C.c_int64, C.c_uint64, C.c_uint32
        L.dblp_embed.argtypes = [vp, i64, u64, u32, C.c_int, vp, u32, u64, i64, C.c_float, vp, i64, C.c_int, vp, vp]
        L.dblp_embed_grad_workspace_bytes.argtypes = [u64, u64, u32, C.POINTER(C.c_size_t)]
        L.dblp_embed_grad.argtypes = [vp, i64, C.c_int, vp, u32, u64, i64, C.c_float, vp, i64, u64, u32, C.c_int, u32, vp, vp,
                                      C.c_size_t, vp]
        L.dblp_dropout.argtypes = [vp, i64, vp, i64, vp, i64, u64, u32, C.c_int, C.c_double, u64, u32, u32, vp]
        L.dblp_dropout_grad.argtypes = [vp, i64, vp, i64, u64, u32, C.c_int, C.c_double, u64, u32, u32, vp]
        at, hd, sz = C.POINTER(dblp_attention_t), C.POINTER(dblp_heads_t), C.POINTER(C.c_size_t)
        L.dblp_attention_workspace_bytes.argtypes = [at, sz, sz]
        L.dblp_attention.argtypes = [at, hd, hd, hd, hd, vp, vp, C.c_size_t, vp]
        L.dblp_attention_grad.argtypes = [at] + [hd] * 5 + [vp] + [hd] * 3 + [vp, C.c_size_t, vp]
        nr, ln, mx, og = (C.POINTER(t) for t in (dblp_norm_rotate_t, dblp_linear_t, dblp_matrix_t, dblp_orthogonalize_t))
        L.dblp_norm_rotate.argtypes = [nr, hd, vp, hd, hd, vp, hd, vp]
        L.dblp_norm_rotate_grad_workspace_bytes.argtypes = [nr, sz]
        L.dblp_norm_rotate_grad.argtypes = [nr, hd, vp, hd, hd, vp, hd, vp, hd, hd, vp, vp, C.c_size_t, vp]
        L.dblp_linear_workspace_bytes.argtypes = [ln, mx, mx, mx, sz, sz]
        L.dblp_linear.argtypes = [ln, mx, mx, vp, mx, mx, mx, vp, C.c_size_t, vp]
        L.dblp_linear_grad.argtypes = [ln] + [mx] * 7 + [vp, vp, C.c_size_t, vp]
        L.dblp_orthogonalize_workspace_bytes.argtypes = [og, sz]
        L.dblp_orthogonalize.argtypes = [og, vp, vp, vp, C.c_size_t, vp]
        _lib = L
    return _lib


def _ptr(t):
    if t is None:
        return C.c_void_p(0)
    if isinstance(t, torch.Tensor):
        assert t.is_contiguous()
        return C.c_void_p(t.data_ptr())
    return C.c_void_p(int(t))


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _check(rc, what):
    if rc != 0:
        raise DblpError(rc, what)


def loss_model(kind, **fields):
    m = dblp_loss_model_t()
    m.kind = LOSS_KINDS[kind] if isinstance(kind, str) else int(kind)
    for k, v in fields.items():
        setattr(m, k, int(v))
    return m


def dblp_loss_model_from_rates(kind, mean_loss=0.0, mean_burst_len=20.0, window_frac=0.05, p_in=0.3, p_out=0.001, C_=0):
    m = dblp_loss_model_t()
    _check(lib().dblp_loss_model_from_rates(LOSS_KINDS[kind] if isinstance(kind, str) else kind, mean_loss,
                                            mean_burst_len, window_frac, p_in, p_out, C_, C.byref(m)),
           "dblp_loss_model_from_rates")
    return m


class Plan:
    """Owns a dblp_plan_t.  Create it with the CUDA device that holds the buffers current."""

    def __init__(self, tensor_numel, dtype, payload_bytes, W, bucket_seq_bounds=None):
        numel = (C.c_uint64 * len(tensor_numel))(*[int(n) for n in tensor_numel])
        dt = {"f32": DBLP_F32, "bf16": DBLP_BF16}[dtype] if isinstance(dtype, str) else int(dtype)
        if bucket_seq_bounds is None:
            bb, B = None, 1
        else:
            bb, B = (C.c_uint64 * len(bucket_seq_bounds))(*[int(b) for b in bucket_seq_bounds]), len(bucket_seq_bounds) - 1
        self.handle = C.c_void_p()
        _check(lib().dblp_plan_create(numel, C.c_uint32(len(tensor_numel)), C.c_int(dt), C.c_uint32(payload_bytes),
                                      C.c_uint32(W), bb, C.c_uint32(B), C.byref(self.handle)), "dblp_plan_create")
        c, n, m, rw = C.c_uint64(), C.c_uint64(), C.c_uint64(), C.c_uint64()
        _check(lib().dblp_plan_query(self.handle, C.byref(c), C.byref(n), C.byref(m), C.byref(rw)), "dblp_plan_query")
        self.C, self.N, self.M, self.row_words = int(c.value), int(n.value), int(m.value), int(rw.value)
        self.T, self.W, self.B, self.P = len(tensor_numel), int(W), B, int(payload_bytes)
        self.es = 4 if dt == DBLP_F32 else 2
        self.torch_dtype = torch.float32 if dt == DBLP_F32 else torch.bfloat16
        ws = C.c_size_t()
        _check(lib().dblp_workspace_bytes(self.handle, C.byref(ws)), "dblp_workspace_bytes")
        self.workspace_bytes = int(ws.value)

    def set_wire_format(self, datagrams):
        """True: one ring of (32 + P)-byte datagrams (pass it as both hdr_ring and payload_ring); False: two rings."""
        _check(lib().dblp_plan_set_wire_format(self.handle, C.c_int(1 if datagrams else 0)), "dblp_plan_set_wire_format")
        self.datagrams = bool(datagrams)

    def set_shard(self, stream_chunks, seq_offset):
        """This plan is the chunks seq_offset .. seq_offset + C - 1 of worker streams of stream_chunks chunks."""
        _check(lib().dblp_plan_set_shard(self.handle, C.c_uint64(stream_chunks), C.c_uint64(seq_offset)), "dblp_plan_set_shard")
        ws = C.c_size_t()
        _check(lib().dblp_workspace_bytes(self.handle, C.byref(ws)), "dblp_workspace_bytes")
        self.workspace_bytes = int(ws.value)

    def tune_reduce(self, chunks_per_tile=0, grid_blocks=0):
        _check(lib().dblp_plan_tune_reduce(self.handle, C.c_uint32(chunks_per_tile), C.c_uint32(grid_blocks)),
               "dblp_plan_tune_reduce")

    def close(self):
        if self.handle:
            lib().dblp_plan_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def alloc_round(self, device, n_slots=None, arrival_cap=None):
        """Device buffers of one round, sized from the plan (torch is the allocator)."""
        n_slots = self.M if n_slots is None else n_slots
        cap = self.M if arrival_cap is None else arrival_cap
        stop_ws = C.c_size_t()
        _check(lib().dblp_stop_workspace_bytes(self.handle, C.c_uint64(cap), C.byref(stop_ws)), "dblp_stop_workspace_bytes")
        claim_ws = C.c_size_t()
        _check(lib().dblp_claim_workspace_bytes(self.handle, C.c_uint64(n_slots), C.c_uint64(cap), C.byref(claim_ws)),
               "dblp_claim_workspace_bytes")
        ws_bytes = max(self.workspace_bytes, int(stop_ws.value), int(claim_ws.value))
        u8, u32, i64 = torch.uint8, torch.int32, torch.int64
        z = lambda n, dt: torch.zeros(n, dtype=dt, device=device)
        return {
            "hdr_ring": z(n_slots * HDR_BYTES, u8), "payload_ring": torch.empty(n_slots * self.P, dtype=u8, device=device),
            "delivered_bits": z(self.W * self.row_words, u32), "arrival": z(cap, u32), "n_arrived": z(1, i64),
            "recv_bitmap": z(self.W * self.row_words, u32), "slot_key": z(self.W * self.C, i64),
            "counters": z(7, i64), "agg": torch.empty(self.N, dtype=torch.float32, device=device),
            "recv_cnt": z(self.W * self.B, u32), "missing_cnt": z(self.W * self.B, u32),
            "ok": z(self.W * self.B, u8), "all_ok": z(1, u32),
            "ws": z((ws_bytes + 7) // 8, i64), "sent_bits": z(self.W * self.row_words, u32),
            "n_slots": n_slots, "arrival_cap": cap,
        }


def dblp_packetize(plan, grads, round, hdr_ring, payload_ring, stream=None):
    ptrs = (C.c_void_p * plan.W)(*[g.data_ptr() for g in grads])
    _check(lib().dblp_packetize(plan.handle, ptrs, C.c_uint32(round), _ptr(hdr_ring), _ptr(payload_ring),
                                _stream(stream)), "dblp_packetize")


def dblp_apply_loss(plan, model, seed, round, attempt, delivered_bits, arrival, n_arrived_dev, ws, stream=None):
    _check(lib().dblp_apply_loss(plan.handle, C.byref(model), C.c_uint64(seed), C.c_uint32(round), C.c_uint32(attempt),
                                 _ptr(delivered_bits), _ptr(arrival), _ptr(n_arrived_dev), _ptr(ws),
                                 C.c_size_t(ws.numel() * ws.element_size()), _stream(stream)), "dblp_apply_loss")


STATIC_SCRATCH_BYTES = 4 * 1024 * 1024 + 64 * 1024


def dblp_apply_loss_static(plan, model, seed, round, attempt, delivered_bits, arrival, n_arrived_dev, stream=None):
    """dblp_apply_loss for callers that may not allocate device memory: the scratch is a fixed array inside the
    library (plans up to STATIC_SCRATCH_BYTES of workspace).  All calls on a device share that array, so calls that
    could overlap on the GPU must be ordered by the caller."""
    _check(lib().dblp_apply_loss_static(plan.handle, C.byref(model), C.c_uint64(seed), C.c_uint32(round),
                                        C.c_uint32(attempt), _ptr(delivered_bits), _ptr(arrival), _ptr(n_arrived_dev),
                                        _stream(stream)), "dblp_apply_loss_static")


def dblp_missing_bits(plan, recv_bitmap, sent_bits, stream=None):
    _check(lib().dblp_missing_bits(plan.handle, _ptr(recv_bitmap), _ptr(sent_bits), _stream(stream)), "dblp_missing_bits")


def dblp_apply_loss_resend(plan, model, seed, round, attempt, sent_bits, delivered_bits, arrival, n_arrived_dev, ws,
                           stream=None):
    _check(lib().dblp_apply_loss_resend(plan.handle, C.byref(model), C.c_uint64(seed), C.c_uint32(round),
                                        C.c_uint32(attempt), _ptr(sent_bits), _ptr(delivered_bits), _ptr(arrival),
                                        _ptr(n_arrived_dev), _ptr(ws), C.c_size_t(ws.numel() * ws.element_size()),
                                        _stream(stream)), "dblp_apply_loss_resend")


def dblp_aggregate_book_stop(plan, hdr_ring, n_slots, arrival, n_arrived_dev, arrival_cap, round, bound_ppm,
                             recv_bitmap, slot_key, counters, ws, stream=None):
    _check(lib().dblp_aggregate_book_stop(plan.handle, _ptr(hdr_ring), C.c_uint64(n_slots), _ptr(arrival),
                                          _ptr(n_arrived_dev), C.c_uint64(arrival_cap), C.c_uint32(round),
                                          C.c_uint32(bound_ppm), _ptr(recv_bitmap), _ptr(slot_key), _ptr(counters),
                                          _ptr(ws), C.c_size_t(ws.numel() * ws.element_size()), _stream(stream)),
           "dblp_aggregate_book_stop")


def _device_buffers(dev, grads_dev=None):
    b = dblp_device_buffers_t()
    b.grads = grads_dev.data_ptr() if grads_dev is not None else 0
    for name in ("hdr_ring", "payload_ring", "delivered_bits", "arrival", "n_arrived", "recv_bitmap", "slot_key",
                 "counters", "agg", "recv_cnt", "missing_cnt", "ok", "all_ok", "ws", "sent_bits"):
        setattr(b, name, dev[name].data_ptr())
    b.ws_bytes = dev["ws"].numel() * dev["ws"].element_size()
    return b


def dblp_round_until_stop(plan, model, seed, round, bound_ppm, max_attempts, early_stop, dev, stream=None):
    """Returns (attempts used, all_ok).  Blocks: the decision is read back after every attempt."""
    b = _device_buffers(dev)
    attempts, ok = C.c_uint32(), C.c_uint32()
    _check(lib().dblp_round_until_stop(plan.handle, C.byref(model), C.c_uint64(seed), C.c_uint32(round),
                                       C.c_uint32(bound_ppm), C.c_uint32(max_attempts), C.c_int(int(early_stop)),
                                       C.byref(b), C.byref(attempts), C.byref(ok), _stream(stream)),
           "dblp_round_until_stop")
    return int(attempts.value), int(ok.value)


def dblp_aggregate_book(plan, hdr_ring, n_slots, arrival, n_arrived_dev, arrival_cap, round, recv_bitmap, slot_key,
                        counters, stream=None):
    _check(lib().dblp_aggregate_book(plan.handle, _ptr(hdr_ring), C.c_uint64(n_slots), _ptr(arrival),
                                     _ptr(n_arrived_dev), C.c_uint64(arrival_cap), C.c_uint32(round), _ptr(recv_bitmap),
                                     _ptr(slot_key), _ptr(counters), _stream(stream)), "dblp_aggregate_book")


def dblp_aggregate_claim(plan, hdr_ring, n_slots, arrival, n_arrived_dev, arrival_cap, round, slot_key, counters,
                         stream=None):
    _check(lib().dblp_aggregate_claim(plan.handle, _ptr(hdr_ring), C.c_uint64(n_slots), _ptr(arrival), _ptr(n_arrived_dev),
                                      C.c_uint64(arrival_cap), C.c_uint32(round), _ptr(slot_key), _ptr(counters),
                                      _stream(stream)), "dblp_aggregate_claim")


def dblp_aggregate_claim_grouped(plan, hdr_ring, n_slots, arrival, n_arrived_dev, arrival_cap, round, slot_key, counters,
                                 ws, stream=None):
    _check(lib().dblp_aggregate_claim_grouped(plan.handle, _ptr(hdr_ring), C.c_uint64(n_slots), _ptr(arrival),
                                              _ptr(n_arrived_dev), C.c_uint64(arrival_cap), C.c_uint32(round), _ptr(slot_key),
                                              _ptr(counters), _ptr(ws), C.c_size_t(ws.numel() * ws.element_size()),
                                              _stream(stream)), "dblp_aggregate_claim_grouped")


def dblp_aggregate_bitmap(plan, slot_key, n_arrived_dev, arrival_cap, recv_bitmap, counters, stream=None):
    _check(lib().dblp_aggregate_bitmap(plan.handle, _ptr(slot_key), _ptr(n_arrived_dev), C.c_uint64(arrival_cap),
                                       _ptr(recv_bitmap), _ptr(counters), _stream(stream)), "dblp_aggregate_bitmap")


def dblp_aggregate_reduce(plan, payload_ring, slot_key, agg_out, flags=DBLP_SUM, stream=None):
    _check(lib().dblp_aggregate_reduce(plan.handle, _ptr(payload_ring), _ptr(slot_key), _ptr(agg_out),
                                       C.c_uint32(flags), _stream(stream)), "dblp_aggregate_reduce")


def dblp_aggregate_reduce_atomic(plan, payload_ring, slot_key, agg_out, flags=DBLP_SUM, stream=None):
    _check(lib().dblp_aggregate_reduce_atomic(plan.handle, _ptr(payload_ring), _ptr(slot_key), _ptr(agg_out),
                                              C.c_uint32(flags), _stream(stream)), "dblp_aggregate_reduce_atomic")


def dblp_norm_scratch_count(plan):
    n = C.c_uint64()
    _check(lib().dblp_norm_scratch_count(plan.handle, C.byref(n)), "dblp_norm_scratch_count")
    return int(n.value)


def dblp_aggregate_reduce_ex(plan, payload_ring, slot_key, agg_out, flags=DBLP_SUM, norm_scratch=None, norm_out=None,
                             params=None, lr=0.0, stream=None):
    _check(lib().dblp_aggregate_reduce_ex(plan.handle, _ptr(payload_ring), _ptr(slot_key), _ptr(agg_out),
                                          C.c_uint32(flags), _ptr(norm_scratch), _ptr(norm_out), _ptr(params),
                                          C.c_float(lr), _stream(stream)), "dblp_aggregate_reduce_ex")


def dblp_aggregate(plan, hdr_ring, payload_ring, n_slots, arrival, n_arrived_dev, arrival_cap, round, recv_bitmap,
                   slot_key, counters, agg_out, flags=DBLP_SUM, stream=None):
    _check(lib().dblp_aggregate(plan.handle, _ptr(hdr_ring), _ptr(payload_ring), C.c_uint64(n_slots), _ptr(arrival),
                                _ptr(n_arrived_dev), C.c_uint64(arrival_cap), C.c_uint32(round), _ptr(recv_bitmap),
                                _ptr(slot_key), _ptr(counters), _ptr(agg_out), C.c_uint32(flags), _stream(stream)),
           "dblp_aggregate")


def dblp_round_reset(plan, recv_bitmap, slot_key, counters, stream=None):
    _check(lib().dblp_round_reset(plan.handle, _ptr(recv_bitmap), _ptr(slot_key), _ptr(counters), _stream(stream)),
           "dblp_round_reset")


def dblp_check_bound(plan, recv_bitmap, bound_ppm, recv_cnt, missing_cnt, ok, all_ok, stream=None):
    bounds = [int(bound_ppm)] if isinstance(bound_ppm, int) else [int(b) for b in bound_ppm]
    arr = (C.c_uint32 * len(bounds))(*bounds)
    _check(lib().dblp_check_bound(plan.handle, _ptr(recv_bitmap), arr, C.c_uint32(len(bounds)), _ptr(recv_cnt),
                                  _ptr(missing_cnt), _ptr(ok), _ptr(all_ok), _stream(stream)), "dblp_check_bound")


def dblp_bound_ok(missing, total, bound_ppm):
    return bool(lib().dblp_bound_ok(C.c_uint64(missing), C.c_uint64(total), C.c_uint32(bound_ppm)))


def dblp_clr(norm_prev, norm_curr, eta=0.5):
    return bool(lib().dblp_clr(norm_prev, norm_curr, eta))


def dblp_select_bound(norm_prev, norm_curr, eta, p_low_ppm, p_high_ppm, at_epoch_start, first_iteration, current_ppm):
    return int(lib().dblp_select_bound(norm_prev, norm_curr, eta, p_low_ppm, p_high_ppm, int(at_epoch_start),
                                       int(first_iteration), current_ppm))


def _marks(marks):
    return C.byref(marks.struct) if marks is not None else None


def _grad_ptrs(plan, grads):
    return (C.c_void_p * plan.W)(*[g.data_ptr() for g in grads])


def dblp_round_send(plan, grads, model, seed, round, dev, marks=None, stream=None):
    b = _device_buffers(dev)
    _check(lib().dblp_round_send(plan.handle, _grad_ptrs(plan, grads), C.byref(model), C.c_uint64(seed), C.c_uint32(round),
                                 C.byref(b), _marks(marks), _stream(stream)), "dblp_round_send")


def dblp_round_receive(plan, round, bound_ppm, flags, dev, marks=None, stream=None):
    b = _device_buffers(dev)
    _check(lib().dblp_round_receive(plan.handle, C.c_uint32(round), C.c_uint32(bound_ppm), C.c_uint32(flags), C.byref(b),
                                    _marks(marks), _stream(stream)), "dblp_round_receive")


def dblp_round_device(plan, grads, model, seed, round, bound_ppm, flags, dev, marks=None, stream=None):
    """One whole round on device-resident gradients with the library's two-stream schedule."""
    b = _device_buffers(dev)
    _check(lib().dblp_round_device(plan.handle, _grad_ptrs(plan, grads), C.byref(model), C.c_uint64(seed),
                                   C.c_uint32(round), C.c_uint32(bound_ppm), C.c_uint32(flags), C.byref(b),
                                   _marks(marks), _stream(stream)), "dblp_round_device")


def dblp_round_host(plan, grads_host, model, seed, round, bound_ppm, flags, dev, grads_dev, agg_host=None,
                    counters_host=None, recv_cnt_host=None, missing_cnt_host=None, ok_host=None, all_ok_host=None,
                    stream=None):
    """grads_host: W host tensors (pinned recommended); dev: buffers from Plan.alloc_round; grads_dev: one device
    tensor of W*N elements; *_host: host tensors that receive the results (None to skip)."""
    ptrs = (C.c_void_p * plan.W)(*[g.data_ptr() for g in grads_host])
    b = _device_buffers(dev, grads_dev)
    _check(lib().dblp_round_host(plan.handle, ptrs, C.byref(model), C.c_uint64(seed), C.c_uint32(round),
                                 C.c_uint32(bound_ppm), C.c_uint32(flags), C.byref(b), _ptr(agg_host),
                                 _ptr(counters_host), _ptr(recv_cnt_host), _ptr(missing_cnt_host), _ptr(ok_host),
                                 _ptr(all_ok_host), _stream(stream)), "dblp_round_host")


# ---- worker side -----------------------------------------------------------------------------------------------------
_DTYPES = {torch.float32: DBLP_F32, torch.bfloat16: DBLP_BF16, torch.float16: DBLP_F16}


def _dtype(t):
    if t.dtype not in _DTYPES:
        raise ValueError("dtype %s: float32, bfloat16 or float16" % t.dtype)
    return _DTYPES[t.dtype]


def _on_device(*tensors):
    """The library launches on the current device: every tensor has to be there."""
    cur = -1
    for t in tensors:
        if t is not None:
            dev = t.get_device()
            if cur < 0 <= dev:
                cur = torch._C._cuda_getDevice()
            if dev < 0 or dev != cur:
                raise ValueError("a tensor on %s, which is not the current device" % t.device)


def _raw_stream(stream):
    """The stream's handle as a number; the current stream's without building a torch.cuda.Stream."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _require(ok, what):
    if not ok:
        raise ValueError(what)


def _u32(x, name):
    """x itself where it fits the 32 bits that the call has for it (a larger one would arrive cut off)."""
    if not 0 <= x < 1 << 32:
        raise ValueError("%s = %d does not fit in 32 bits" % (name, x))
    return x


def _rows(t, name):
    """(address, row stride, rows, columns) of a 2-D tensor whose elements within a row are contiguous."""
    if t.dim() != 2:
        raise ValueError("%s: 2-D" % name)
    (rows, cols), (rs, cs) = t.shape, t.stride()
    if cs != 1 and cols > 1:
        raise ValueError("%s: contiguous within a row" % name)
    return t.data_ptr(), rs, rows, cols


_TOKEN_BYTES = {torch.int32: 4, torch.int64: 8}


def _flat_tokens(tokens):
    b = _TOKEN_BYTES.get(tokens.dtype)
    if b is None or tokens.dim() != 1 or not tokens.is_contiguous():
        raise ValueError("tokens: 1-D, contiguous, int32 or int64")
    return tokens.data_ptr(), b, tokens.shape[0]


def _counter(t):
    if t is None:
        return None
    _require(t.dtype == torch.int64 and t.numel() == 1, "bad_tokens: one int64")
    return t.data_ptr()


def _scratch(ws):
    if ws is None or ws.numel() == 0:
        return None, 0
    _require(ws.is_contiguous(), "workspace: contiguous")
    return ws.data_ptr(), ws.nbytes


def dblp_embed(table, tokens, out, scale=1.0, padding=-1, bad_tokens=None, stream=None):
    """out[i] = scale * table[tokens[i]]; a zero row for the padding id (none if outside the table) and for ids outside the
    table, which bad_tokens counts."""
    _on_device(table, tokens, out, bad_tokens)
    tp, ts, rows, width = _rows(table, "table")
    op, os_, m, w = _rows(out, "out")
    kp, kb, n = _flat_tokens(tokens)
    if m != n or w != width:
        raise ValueError("out: one row of the table's width per token")
    _check(lib().dblp_embed(tp, ts, rows, _u32(width, "width"), _dtype(table), kp, kb, n, padding, scale, op, os_, _dtype(out),
                            _counter(bad_tokens), _raw_stream(stream)), "dblp_embed")


def dblp_embed_grad_workspace_bytes(n, rows, width):
    b = C.c_size_t()
    _check(lib().dblp_embed_grad_workspace_bytes(n, rows, _u32(width, "width"), C.byref(b)), "dblp_embed_grad_workspace_bytes")
    return int(b.value)


def dblp_embed_grad(dout, tokens, dtable, ws, scale=1.0, padding=-1, accumulate=False, bad_tokens=None, stream=None):
    """dtable[v] = scale * sum of dout[i] over the i with tokens[i] = v (added to dtable with accumulate)."""
    _on_device(dout, tokens, dtable, ws, bad_tokens)
    dp, ds, m, w = _rows(dout, "dout")
    tp, ts, rows, width = _rows(dtable, "dtable")
    kp, kb, n = _flat_tokens(tokens)
    if m != n or w != width:
        raise ValueError("dout: one row of the table's width per token")
    wp, wb = _scratch(ws)
    _check(lib().dblp_embed_grad(dp, ds, _dtype(dout), kp, kb, n, padding, scale, tp, ts, rows, _u32(width, "width"), _dtype(dtable),
                                 DBLP_ACCUMULATE if accumulate else 0, _counter(bad_tokens), wp, wb, _raw_stream(stream)),
           "dblp_embed_grad")


def dblp_dropout(x, out, p, seed, step, site, residual=None, stream=None):
    """out = dropout(x) [+ residual]; (seed, step, site) names the mask."""
    _on_device(x, out, residual)
    xp, xs, rows, cols = _rows(x, "x")
    op, os_, m, w = _rows(out, "out")
    rp = rs = None
    same = m == rows and w == cols and out.dtype == x.dtype
    if residual is not None:
        rp, rs, m, w = _rows(residual, "residual")
        same = same and m == rows and w == cols and residual.dtype == x.dtype
    if not same:
        raise ValueError("x, residual and out: one shape and dtype")
    _check(lib().dblp_dropout(xp, xs, rp, rs or 0, op, os_, rows, _u32(cols, "columns"), _dtype(x), p, seed, _u32(step, "step"),
                              _u32(site, "site"), _raw_stream(stream)), "dblp_dropout")


def dblp_dropout_grad(dout, dx, p, seed, step, site, stream=None):
    """Gradient of dblp_dropout's x: the mask of (seed, step, site) drawn again."""
    _on_device(dout, dx)
    gp, gs, rows, cols = _rows(dout, "dout")
    xp, xs, m, w = _rows(dx, "dx")
    if m != rows or w != cols or dx.dtype != dout.dtype:
        raise ValueError("dout and dx: one shape and dtype")
    _check(lib().dblp_dropout_grad(gp, gs, xp, xs, rows, _u32(cols, "columns"), _dtype(dx), p, seed, _u32(step, "step"),
                                   _u32(site, "site"), _raw_stream(stream)), "dblp_dropout_grad")


def _heads(t, name, dtype, shape):
    if t.dtype != dtype or t.shape != shape:
        raise ValueError("%s: shape %s, %s" % (name, shape, dtype))
    sb, st, sh, sd = t.stride()
    if sd != 1 and shape[3] > 1:
        raise ValueError("%s: the elements of a head are contiguous" % name)
    return C.byref(dblp_heads_t(t.data_ptr(), sb, st, sh))


def _attention(q, k, causal, scale, q_lens, k_lens):
    """(the call's description, q's shape, k's shape)"""
    _require(q.dim() == 4 and k.dim() == 4, "q and k: [batch, tokens, heads, head_dim]")
    qs, ks = q.shape, k.shape
    B, Sq, Hq, D = qs
    _require(ks[0] == B and ks[3] == D, "q and k: one batch and head_dim")
    for n in (q_lens, k_lens):
        if n is not None and not (n.dtype == torch.int32 and n.shape == (B,) and n.is_contiguous()):
            raise ValueError("lengths: int32, one per sequence")
    if scale is None:
        scale = D ** -0.5 if D else 0.0
    if max(B, Sq, ks[1], Hq, ks[2], D) >= 1 << 32:
        raise ValueError("an extent of q or k does not fit in 32 bits")
    return dblp_attention_t(B, Sq, ks[1], Hq, ks[2], D, _dtype(q), DBLP_ATTENTION_CAUSAL if causal else 0, scale,
                            None if q_lens is None else q_lens.data_ptr(), None if k_lens is None else k_lens.data_ptr()), qs, ks


def _lse(lse, qs):
    if lse.dtype != torch.float32 or lse.shape != (qs[0], qs[2], qs[1]) or not lse.is_contiguous():
        raise ValueError("lse: contiguous float32 [batch, heads, tokens]")
    return lse.data_ptr()


def dblp_attention_workspace_bytes(q, k, causal=False):
    """(bytes for dblp_attention, bytes for dblp_attention_grad) with tensors of these shapes."""
    f, g = C.c_size_t(), C.c_size_t()
    _check(lib().dblp_attention_workspace_bytes(C.byref(_attention(q, k, causal, None, None, None)[0]), C.byref(f), C.byref(g)),
           "dblp_attention_workspace_bytes")
    return int(f.value), int(g.value)


def dblp_attention(q, k, v, out, lse=None, ws=None, causal=False, scale=None, q_lens=None, k_lens=None, stream=None):
    """q, out [batch, tokens, heads, head_dim]; k, v [batch, keys, key heads, head_dim]; lse fp32 [batch, heads, tokens]."""
    _on_device(q, k, v, out, lse, ws, q_lens, k_lens)
    a, qs, ks = _attention(q, k, causal, scale, q_lens, k_lens)
    dt = q.dtype
    wp, wb = _scratch(ws)
    _check(lib().dblp_attention(C.byref(a), _heads(q, "q", dt, qs), _heads(k, "k", dt, ks), _heads(v, "v", dt, ks),
                                _heads(out, "out", dt, qs), None if lse is None else _lse(lse, qs), wp, wb, _raw_stream(stream)),
           "dblp_attention")


def dblp_attention_grad(q, k, v, out, dout, lse, dq, dk, dv, ws, causal=False, scale=None, q_lens=None, k_lens=None,
                        stream=None):
    """Gradients of dblp_attention, from its inputs, its out and lse, and dout."""
    _on_device(q, k, v, out, dout, lse, dq, dk, dv, ws, q_lens, k_lens)
    a, qs, ks = _attention(q, k, causal, scale, q_lens, k_lens)
    dt = q.dtype
    wp, wb = _scratch(ws)
    _check(lib().dblp_attention_grad(C.byref(a), _heads(q, "q", dt, qs), _heads(k, "k", dt, ks), _heads(v, "v", dt, ks),
                                     _heads(out, "out", dt, qs), _heads(dout, "dout", dt, qs), _lse(lse, qs),
                                     _heads(dq, "dq", dt, qs), _heads(dk, "dk", dt, ks), _heads(dv, "dv", dt, ks), wp, wb,
                                     _raw_stream(stream)), "dblp_attention_grad")


def _norm_rotate(q, k, q_weight, k_weight, positions, freqs, eps, flags):
    """(the call's description, q's shape, k's shape or None); plain comparisons, since a call of a few tokens waits for them"""
    qs, ks, dt = q.shape, None if k is None else k.shape, q.dtype
    if len(qs) != 4 or (ks is not None and len(ks) != 4):
        raise ValueError("q and k: [batch, tokens, heads, head_dim]")
    B, T, Hq, D = qs
    Hk = 0
    if ks is not None:
        if ks[0] != B or ks[1] != T or ks[3] != D or k.dtype is not dt:
            raise ValueError("q and k: one batch, length, head_dim and dtype")
        Hk = ks[2]
    w = q_weight if q_weight is not None else k_weight
    if w is not None:
        wt = w.dtype
        for t in (q_weight, k_weight):
            if t is not None and (t.dtype is not wt or t.dim() != 1 or t.shape[0] != D or not t.is_contiguous()):
                raise ValueError("weights: contiguous, one per column of a head, of one dtype")
    if B >= 1 << 32 or T >= 1 << 32 or Hq >= 1 << 32 or D >= 1 << 32 or Hk >= 1 << 32:
        raise ValueError("an extent of q or k does not fit in 32 bits")
    n = 0 if freqs is None else freqs.numel()
    pp = fp = None
    stride = 0
    if n:
        if freqs.dtype is not torch.float64 or freqs.dim() != 1 or not freqs.is_contiguous():
            raise ValueError("freqs: 1-D, contiguous, float64")
        if positions is None or positions.dtype is not torch.int32 or positions.shape != (B, T) or (T > 1 and positions.stride(1) != 1):
            raise ValueError("positions: int32 [batch, tokens], the tokens of a sequence contiguous")
        pp, fp, stride = positions.data_ptr(), freqs.data_ptr(), positions.stride(0)
    return dblp_norm_rotate_t(B, T, Hq, Hk, D, _u32(2 * n, "rotary_dim"), _dtype(q), DBLP_F32 if w is None else _dtype(w), flags, eps, pp,
                              stride, fp), qs, ks


def _address(t):
    return None if t is None else t.data_ptr()


def _pair(t, name, dtype, shape):
    if shape is None:
        _require(t is None, "%s: there is no k" % name)
        return None
    _require(t is not None, "%s: missing" % name)
    return _heads(t, name, dtype, shape)


def dblp_norm_rotate(q, k, q_weight, k_weight, positions, freqs, q_out, k_out, eps=1e-6, interleaved=False, stream=None):
    """Norm of every head of q and k [batch, tokens, heads, head_dim] and rotation of the first 2 len(freqs) columns by
    positions [batch, tokens] (int32) times freqs (float64, radians a position).  k, k_weight and k_out may be None; weights None
    = ones; freqs None = no rotation."""
    _on_device(q, k, q_weight, k_weight, positions, freqs, q_out, k_out)
    a, qs, ks = _norm_rotate(q, k, q_weight, k_weight, positions, freqs, eps, DBLP_ROTATE_INTERLEAVED if interleaved else 0)
    dt = q.dtype
    _check(lib().dblp_norm_rotate(C.byref(a), _heads(q, "q", dt, qs), _address(q_weight), _heads(q_out, "q_out", dt, qs),
                                  _pair(k, "k", dt, ks), _address(k_weight), _pair(k_out, "k_out", dt, ks), _raw_stream(stream)),
           "dblp_norm_rotate")


def dblp_norm_rotate_grad_workspace_bytes(q, k):
    b = C.c_size_t()
    a = _norm_rotate(q, k, None, None, None, None, 1.0, 0)[0]
    _check(lib().dblp_norm_rotate_grad_workspace_bytes(C.byref(a), C.byref(b)), "dblp_norm_rotate_grad_workspace_bytes")
    return int(b.value)


def dblp_norm_rotate_grad(q, k, q_weight, k_weight, positions, freqs, dq_out, dk_out, dq, dk, dq_weight=None, dk_weight=None,
                          ws=None, eps=1e-6, interleaved=False, accumulate=False, stream=None):
    """Gradients of dblp_norm_rotate's q, k and weights, from its inputs and the gradients of its outputs."""
    _on_device(q, k, q_weight, k_weight, positions, freqs, dq_out, dk_out, dq, dk, dq_weight, dk_weight, ws)
    flags = (DBLP_ROTATE_INTERLEAVED if interleaved else 0) | (DBLP_ACCUMULATE if accumulate else 0)
    a, qs, ks = _norm_rotate(q, k, q_weight, k_weight, positions, freqs, eps, flags)
    dt = q.dtype
    for t in (dq_weight, dk_weight):
        if t is None:
            continue
        if q_weight is None and k_weight is None:
            _require(dq_weight is None or dk_weight is None or dq_weight.dtype == dk_weight.dtype, "gradients of the weights: one dtype")
            a.weight_dtype = _dtype(t)
        elif _dtype(t) != a.weight_dtype:
            raise ValueError("gradients of the weights: the weights' dtype")
        _require(t.shape == (qs[3],) and t.is_contiguous(), "gradients of the weights: contiguous, one per column of a head")
    wp, wb = _scratch(ws)
    _check(lib().dblp_norm_rotate_grad(C.byref(a), _heads(q, "q", dt, qs), _address(q_weight), _heads(dq_out, "dq_out", dt, qs),
                                       _heads(dq, "dq", dt, qs), _address(dq_weight), _pair(k, "k", dt, ks), _address(k_weight),
                                       _pair(dk_out, "dk_out", dt, ks), _pair(dk, "dk", dt, ks), _address(dk_weight), wp, wb,
                                       _raw_stream(stream)), "dblp_norm_rotate_grad")


def _matrix(t, name, rows, cols, dtype):
    if t.shape != (rows, cols) or t.dtype != dtype:
        raise ValueError("%s: %d x %d, %s" % (name, rows, cols, dtype))
    rs, cs = t.stride()
    return C.byref(dblp_matrix_t(t.data_ptr(), rs, cs))


def _activation(name):
    if name not in ACTIVATIONS:
        raise ValueError("activation %r: one of %s" % (name, ", ".join(map(repr, ACTIVATIONS))))
    return ACTIVATIONS[name]


def _linear(x, w, out_dtype, bias, activation, flags):
    xs, ws, dt = x.shape, w.shape, x.dtype
    if len(xs) != 2 or len(ws) != 2 or xs[1] != ws[0]:
        raise ValueError("x and w: rows x in, in x out")
    (n, i), o = xs, ws[1]
    if w.dtype is not dt:
        raise ValueError("x and w: one dtype")
    if n >= 1 << 32 or i >= 1 << 32 or o >= 1 << 32:
        raise ValueError("an extent does not fit in 32 bits")
    if bias is not None and (bias.dim() != 1 or bias.shape[0] != o or not bias.is_contiguous()):
        raise ValueError("bias and its gradient: contiguous, one per column of w")
    code = _dtype(x)
    return dblp_linear_t(n, i, o, code, code if out_dtype is None else _DTYPES.get(out_dtype, -1), DBLP_F32 if bias is None else _dtype(bias),
                         _activation(activation), flags), n, i, o


def dblp_linear_workspace_bytes(x, w, dy=None):
    """(bytes for dblp_linear, bytes for dblp_linear_grad) with these tensors; the second is 0 without dy."""
    l, n, i, o = _linear(x, w, None, None, None, 0)
    f, g = C.c_size_t(), C.c_size_t()
    _check(lib().dblp_linear_workspace_bytes(C.byref(l), _matrix(x, "x", n, i, x.dtype), _matrix(w, "w", i, o, x.dtype),
                                             None if dy is None else _matrix(dy, "dy", n, o, x.dtype), C.byref(f), C.byref(g)),
           "dblp_linear_workspace_bytes")
    return int(f.value), int(g.value)


def dblp_linear(x, w, out, ws=None, bias=None, residual=None, pre=None, activation=None, stream=None):
    """out = act(x w + bias) + residual, pre = x w + bias; x [rows, in], w [in, out] (or the transposed view of [out, in])."""
    _on_device(x, w, out, ws, bias, residual, pre)
    l, n, i, o = _linear(x, w, out.dtype, bias, activation, 0)
    dt, od = x.dtype, out.dtype
    wp, wb = _scratch(ws)
    _check(lib().dblp_linear(C.byref(l), _matrix(x, "x", n, i, dt), _matrix(w, "w", i, o, dt), _address(bias),
                             None if residual is None else _matrix(residual, "residual", n, o, od),
                             None if pre is None else _matrix(pre, "pre", n, o, dt), _matrix(out, "out", n, o, od), wp, wb,
                             _raw_stream(stream)), "dblp_linear")


def dblp_linear_grad(dy, x, w, dx=None, dw=None, dbias=None, ws=None, residual=None, pre=None, activation=None, accumulate=False,
                     stream=None):
    """dx = (dy w^T + residual) act'(pre), with pre and the activation those of the layer that made x; dw = x^T dy; dbias = sum of
    dy's rows.  With accumulate, dw and dbias are added to."""
    _on_device(dy, x, w, dx, dw, dbias, ws, residual, pre)
    l, n, i, o = _linear(x, w, None if dw is None else dw.dtype, dbias, activation, DBLP_ACCUMULATE if accumulate else 0)
    dt = x.dtype
    wp, wb = _scratch(ws)
    _check(lib().dblp_linear_grad(C.byref(l), _matrix(dy, "dy", n, o, dt), _matrix(x, "x", n, i, dt), _matrix(w, "w", i, o, dt),
                                  None if residual is None else _matrix(residual, "residual", n, i, dt),
                                  None if pre is None else _matrix(pre, "pre", n, i, dt),
                                  None if dx is None else _matrix(dx, "dx", n, i, dt),
                                  None if dw is None else _matrix(dw, "dw", i, o, dw.dtype), _address(dbias), wp, wb,
                                  _raw_stream(stream)), "dblp_linear_grad")


def _orthogonalize(x, out, coefficients, eps, scale):
    _require(x.dim() in (2, 3) and x.shape == out.shape, "x and out: one shape, [rows, cols] or [batch, rows, cols]")
    b = x.shape[0] if x.dim() == 3 else 1
    m, n = x.shape[-2:]
    if max(b, m, n) >= 1 << 32:
        raise ValueError("an extent does not fit in 32 bits")
    for t, name in ((x, "x"), (out, "out")):
        _require(n <= 1 or t.stride(-1) == 1, "%s: contiguous within a row" % name)
    flat = [float(v) for abc in coefficients for v in abc]
    _require(len(flat) == 3 * len(coefficients), "coefficients: triples (a, b, c)")
    each = [t.stride(0) if x.dim() == 3 else 0 for t in (x, out)]
    return dblp_orthogonalize_t(b, m, n, _dtype(x), _dtype(out), len(coefficients), (C.c_float * max(1, len(flat)))(*flat), eps, scale,
                                each[0], x.stride(-2), each[1], out.stride(-2))


def dblp_orthogonalize_workspace_bytes(x, out):
    b = C.c_size_t()
    a = _orthogonalize(x, out, MUON_COEFFICIENTS, 0.0, 1.0)
    _check(lib().dblp_orthogonalize_workspace_bytes(C.byref(a), C.byref(b)), "dblp_orthogonalize_workspace_bytes")
    return int(b.value)


def dblp_orthogonalize(x, out, ws, coefficients=MUON_COEFFICIENTS, eps=1e-7, scale=1.0, stream=None):
    """out = scale times x with its singular values brought near 1, by one Newton-Schulz product a X + b X X^T X + c (X X^T)^2 X per
    triple; x [rows, cols] or [batch, rows, cols].  out may be x."""
    _on_device(x, out, ws)
    a = _orthogonalize(x, out, coefficients, eps, scale)
    wp, wb = _scratch(ws)
    _check(lib().dblp_orthogonalize(C.byref(a), x.data_ptr(), out.data_ptr(), wp, wb, _raw_stream(stream)), "dblp_orthogonalize")


def dblp_wait_timeouts():
    n = C.c_uint64()
    _check(lib().dblp_wait_timeouts(C.byref(n)), "dblp_wait_timeouts")
    return int(n.value)


def dblp_launch_count():
    return int(lib().dblp_launch_count())


def counters_dict(counters_tensor):
    v = counters_tensor.cpu().tolist()
    d = dict(zip(COUNTER_FIELDS, v[:6]))
    d["status"] = v[6] & 0xFFFFFFFF
    return d
