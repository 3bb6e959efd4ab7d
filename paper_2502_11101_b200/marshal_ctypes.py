"""The calls of csrc/binding.cpp through ctypes: same names, same positional arguments, same results.  binding.py uses them where
the native module has not been built for the running torch and Python; a call takes 6 to 20 us of host time instead of 1 to 5."""
from __future__ import annotations

import ctypes

import torch

from . import binding as B

_ref = ctypes.byref


def _bytes(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


def _require(ok: bool, what: str) -> None:
    if not ok:
        raise AssertionError(what)


def plan_init(geom, batch, plan, order, kept_count, query_start, score_accum, stream):
    return B.load_library().cf_plan_init_scores(_ref(geom), _ref(batch), B._ptr(order), B._ptr(kept_count), query_start,
                                                B._ptr(score_accum), plan.data_ptr(), _bytes(plan), B._stream(stream))


def prune_topk(geom, batch, plan, score_accum, keep, keep_per_request, strategy, stream):
    return B.load_library().cf_prune_topk(_ref(geom), _ref(batch), plan.data_ptr(), score_accum.data_ptr(), keep,
                                          B._ptr(keep_per_request), strategy, B._stream(stream))


def reposition_keys(geom, batch, plan, k_in, k_out, n_layers, layer_stride, stream):
    return B.load_library().cf_reposition_keys(_ref(geom), _ref(batch), plan.data_ptr(), n_layers, layer_stride, k_in.data_ptr(),
                                               k_out.data_ptr(), B._stream(stream))


def query_prefill_attn(geom, batch, plan, q, k, v, out, workspace, lse, doc_scores, score_accum, scale, stream):
    return B.load_library().cf_query_prefill_attn(_ref(geom), _ref(batch), plan.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                                  scale, out.data_ptr(), B._ptr(lse), B._ptr(doc_scores), B._ptr(score_accum),
                                                  workspace.data_ptr(), _bytes(workspace), B._stream(stream))


def query_prefill_attn_slot(geom, batch, plan, slot, n_slots, q, k, v, out, workspace, lse, scale, stream):
    return B.load_library().cf_query_prefill_attn_slot(_ref(geom), _ref(batch), plan.data_ptr(), slot, n_slots, q.data_ptr(),
                                                       k.data_ptr(), v.data_ptr(), scale, out.data_ptr(), B._ptr(lse),
                                                       workspace.data_ptr(), _bytes(workspace), B._stream(stream))


def accumulate_scores(geom, batch, plan, n_filled, n_slots, workspace, doc_scores, score_accum, stream):
    return B.load_library().cf_accumulate_scores(_ref(geom), _ref(batch), plan.data_ptr(), n_filled, n_slots, B._ptr(doc_scores),
                                                 B._ptr(score_accum), workspace.data_ptr(), _bytes(workspace), B._stream(stream))


def assemble_final_cache(geom, batch, plan, k, v, k_self, v_self, k_out, v_out, final_rows, stream):
    _require(k_out.is_contiguous() and v_out.is_contiguous() and k_out.shape == v_out.shape, "k_out and v_out: contiguous, of one shape")
    _require(final_rows.dtype == torch.int32 and k.stride(0) == v.stride(0), "final_rows: int32; k_cache and v_cache: one layer stride")
    return B.load_library().cf_assemble_final_cache(_ref(geom), _ref(batch), plan.data_ptr(), k.shape[0], k.stride(0), k.data_ptr(),
                                                    v.data_ptr(), k_self.stride(0), k_self.data_ptr(), v_self.data_ptr(),
                                                    k_out.shape[2], k_out.data_ptr(), v_out.data_ptr(), final_rows.data_ptr(),
                                                    B._stream(stream))


def document_prefill_attn(geom, doc_offsets, max_doc_len, q, k, v, out, k_prefix, v_prefix, lse, scale, token_stride, status, stream):
    n = q.shape[0]
    _require(doc_offsets.dtype == torch.int32 and doc_offsets.is_contiguous(), "doc_offsets: contiguous int32")
    _require(k.shape[0] == n and v.shape[0] == n and out.shape[0] == n, "q, k, v and out: one number of layers")
    _require(k.stride(0) == v.stride(0) and (lse is None or lse.is_contiguous()), "k and v: one layer stride; lse: contiguous")
    prefix = 0 if k_prefix is None else k_prefix.shape[1]
    _require(prefix == 0 or (v_prefix is not None and k_prefix.stride(0) == v_prefix.stride(0)), "k_prefix and v_prefix: one layer stride")
    docs = B.cf_doc_batch(doc_offsets.numel() - 1, max_doc_len, prefix, 0, q.shape[1],
                          k.shape[2] * k.shape[3] if token_stride is None else token_stride, doc_offsets.data_ptr())
    return B.load_library().cf_document_prefill_attn(_ref(geom), _ref(docs), n, q.data_ptr(), q.stride(0), k.data_ptr(), v.data_ptr(),
                                                     k.stride(0), B._ptr(k_prefix) if prefix else None,
                                                     B._ptr(v_prefix) if prefix else None, k_prefix.stride(0) if prefix else 0, scale,
                                                     out.data_ptr(), out.stride(0), B._ptr(lse), B._ptr(status), B._stream(stream))


def decode_plan(geom, n_requests, cache_rows, rows, extra_rows, plan, stream):
    return B.load_library().cf_decode_plan(_ref(geom), n_requests, cache_rows, rows.data_ptr(), extra_rows, plan.data_ptr(),
                                           _bytes(plan), B._stream(stream))


def decode_attn(geom, n_requests, cache_rows, plan, q, k, v, out, workspace, lse, scale, stream):
    n = q.shape[0]
    _require(k.shape[0] == n and v.shape[0] == n and out.shape[0] == n, "q, k_final, v_final and out: one number of layers")
    _require(k.stride(0) == v.stride(0) and (lse is None or lse.is_contiguous()), "k_final and v_final: one layer stride; lse: contiguous")
    return B.load_library().cf_decode_attn(_ref(geom), n_requests, cache_rows, plan.data_ptr(), n, q.data_ptr(), q.stride(0),
                                           k.data_ptr(), v.data_ptr(), k.stride(0), scale, out.data_ptr(), out.stride(0), B._ptr(lse),
                                           workspace.data_ptr(), _bytes(workspace), B._stream(stream))


def decode_append(geom, n_requests, cache_rows, k, v, rows, step, k_new, v_new, status, stream):
    n = k.shape[0]
    _require(v.shape[0] == n and k_new.shape[0] == n and v_new.shape[0] == n, "k_final, v_final, k_new and v_new: one number of layers")
    _require(k.stride(0) == v.stride(0) and k_new.stride(0) == v_new.stride(0), "keys and values: one layer stride")
    return B.load_library().cf_decode_append(_ref(geom), n_requests, cache_rows, n, k.data_ptr(), v.data_ptr(), k.stride(0),
                                             rows.data_ptr(), step, k_new.data_ptr(), v_new.data_ptr(), k_new.stride(0),
                                             B._ptr(status), B._stream(stream))


def run_stack(geom, batch, plan, workspace, q, k, v, out, score_accum, schedule, strategy, batch_layers, lse, layer_scores, k_final,
              k_self, v_self, scale, doc_len, req_doc_begin, k_prefix, v_prefix, stream):
    stack, keepalive = B.make_stack(q, k, v, out, score_accum, schedule, strategy, batch_layers, lse, layer_scores, k_final, k_self,
                                    v_self, scale, doc_len, req_doc_begin, k_prefix, v_prefix)
    lib = B.load_library()
    need = lib.cf_run_stack_workspace_bytes(_ref(geom), _ref(batch), _ref(stack))
    if need > _bytes(workspace):
        return 0, need
    code = lib.cf_run_stack(_ref(geom), _ref(batch), _ref(stack), plan.data_ptr(), _bytes(plan), workspace.data_ptr(),
                            _bytes(workspace), B._stream(stream))
    del keepalive
    return code, 0


def _require_here(pages, *tensors):
    """The calls below check what they are given: on the current device, whose stream they take."""
    B._pages_here(pages)
    for t in tensors:
        _require(t is None or (t.is_cuda and t.get_device() == torch.cuda.current_device()), "a tensor on the current device is expected")


def _dense_layers(t):
    return t.dim() >= 1 and (t.shape[0] == 0 or t[0].is_contiguous())


def _of_storage_type(geom, t):
    return t.dtype == (torch.bfloat16 if geom.dtype == B.CF_BF16 else torch.float32)


def _require_pool(geom, pages, kv4, layers):
    """A pool of `layers` layers for the pages, each dense."""
    _require(kv4.dtype == torch.uint8 and kv4.dim() >= 1 and kv4.shape[0] == layers and _dense_layers(kv4), "kv4: bytes of as many layers, each dense")
    _require(layers == 0 or kv4.numel() // layers >= B.cf_kv4_layer_bytes(geom, pages), "kv4: fewer bytes than the pages have")


def pages_resize(pages, rows, extra_rows, slots, stream):
    _require(rows.dtype == torch.int32 and rows.is_contiguous() and rows.numel() == pages.n_requests > 0, "rows: int32, one per request")
    _require(slots is None or (slots.dtype == torch.int64 and slots.is_contiguous() and slots.numel() % pages.n_requests == 0),
             "slots: int64, as many for each request")
    _require_here(pages, rows, slots)
    return B.load_library().cf_pages_resize(_ref(pages), rows.data_ptr(), extra_rows, 0 if slots is None else slots.numel() // pages.n_requests,
                                            B._ptr(slots), B._stream(stream))


def _layer_stride(t):
    """Distance between layers, where there are several: a dimension of size 1 may have any stride, nobody steps along it."""
    return t.stride(0) if t.shape[0] > 1 else 0


def _rows_of(geom, t):
    """(layers, rows of a layer, layer stride, row stride) of k or v: rows one behind the other, as far apart as the innermost of
    their dimensions that has several."""
    _require(t.dim() >= 4 and t.shape[-2] == geom.n_kv_heads and t.shape[-1] == geom.head_dim, "k and v: [layers, rows ..., heads, dims]")
    _require(_of_storage_type(geom, t), "k and v: the storage type of the geometry")
    _require(t.stride(-1) == 1 and (t.shape[-2] == 1 or t.stride(-2) == geom.head_dim), "k and v: a row is dense")
    stride, n = geom.n_kv_heads * geom.head_dim, 1
    for d in range(t.dim() - 3, 0, -1):
        if t.shape[d] != 1 and t.numel() != 0:
            if n == 1:
                stride = t.stride(d)
            _require(t.stride(d) == stride * n, "k and v: rows lie one behind the other")
        n *= t.shape[d]
    return t.shape[0], n, _layer_stride(t), stride


def _rows(geom, pages, kv4, slots, k, v):
    rows = _rows_of(geom, k)
    _require(k.shape == v.shape and rows == _rows_of(geom, v), "k and v: one shape and stride")
    _require(slots.dtype == torch.int64 and slots.is_contiguous() and slots.numel() == rows[1], "slots: int64, one per row of a layer")
    _require_pool(geom, pages, kv4, k.shape[0])
    _require_here(pages, kv4, slots, k, v)
    return rows


def kv4_write(geom, pages, kv4, slots, k, v, stream):
    layers, n, layer_stride, stride = _rows(geom, pages, kv4, slots, k, v)
    return B.load_library().cf_kv4_write(_ref(geom), _ref(pages), layers, n, slots.data_ptr(), k.data_ptr(), v.data_ptr(), layer_stride,
                                         stride, kv4.data_ptr(), _layer_stride(kv4), B._stream(stream))


def kv4_read(geom, pages, kv4, slots, k, v, stream):
    layers, n, layer_stride, stride = _rows(geom, pages, kv4, slots, k, v)
    return B.load_library().cf_kv4_read(_ref(geom), _ref(pages), layers, n, slots.data_ptr(), kv4.data_ptr(), _layer_stride(kv4), k.data_ptr(),
                                        v.data_ptr(), layer_stride, stride, B._stream(stream))


def kv4_attn(geom, pages, kv4, q, out, workspace, lse, scale, stream):
    _require(q.dim() == 5 and out.shape == q.shape and q[0].is_contiguous() and out[0].is_contiguous(), "q and out: [layers, requests, tokens, heads, dims]")
    _require(_of_storage_type(geom, q) and _of_storage_type(geom, out), "q and out: the storage type of the geometry")
    _require(q.shape[1] == pages.n_requests and q.shape[3] == geom.n_q_heads and q.shape[4] == geom.head_dim, "q: of other sizes than the geometry and the pages")
    _require(lse is None or (lse.dtype == torch.float32 and lse.is_contiguous() and lse.numel() == q.numel() // geom.head_dim), "lse: fp32, one per query and head")
    _require(workspace.is_contiguous(), "workspace: dense")
    _require_pool(geom, pages, kv4, q.shape[0])
    _require_here(pages, kv4, q, out, workspace, lse)
    return B.load_library().cf_kv4_attn(_ref(geom), _ref(pages), q.shape[0], q.shape[2], q.data_ptr(), _layer_stride(q), kv4.data_ptr(), _layer_stride(kv4),
                                        scale, out.data_ptr(), _layer_stride(out), B._ptr(lse), workspace.data_ptr(), _bytes(workspace), B._stream(stream))
