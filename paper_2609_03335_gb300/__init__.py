"""GB300-native batched evaluation of physical execution plans.

The product is the CUDA library ``libwf.so`` (C ABI in ``include/wf.h``);
``wf`` is its ctypes binding.  Build with ``paper_2609_03335_gb300.build.build()``.
"""
from .wf import (Attn, BeamOut, Ctx, Decode, DevicePlans, Kv, KvLayer, KvMoves, KvStep, Results, Rope, WfError, evaluate, load_library,
                 wf_attend, wf_attn_limit_waits, wf_attn_status, wf_beam_select, wf_ctx_create, wf_ctx_destroy, wf_ctx_status, wf_eval_plans, wf_forecast_readiness, wf_last_error,
                 wf_kv_copy_scales, wf_kv_extend, wf_kv_reorder, wf_kv_write, wf_problem_check, wf_strerror, wf_topk)

__all__ = ["Attn", "BeamOut", "Ctx", "Decode", "DevicePlans", "Kv", "KvLayer", "KvMoves", "KvStep", "Results", "Rope", "WfError", "evaluate",
           "load_library", "wf_attend", "wf_attn_limit_waits", "wf_attn_status", "wf_beam_select", "wf_kv_copy_scales", "wf_kv_extend", "wf_kv_reorder", "wf_kv_write", "wf_ctx_create",
           "wf_ctx_destroy", "wf_ctx_status", "wf_eval_plans", "wf_forecast_readiness",
           "wf_last_error", "wf_problem_check", "wf_strerror", "wf_topk"]
