"""IntentKV per-step retention hot path on MI355X (gfx950).

The HIP library ``libikv.so`` (C ABI in ``include/ikv.h``) holds every step:
QueryMemory update, rule + residual scoring, budgeted selection, slot-map
redirect and slot-map decode attention. This package is its Python binding.
"""
from .ikv import (CALL_CHUNK, CALL_DECODE, CALL_REDIRECT, CALL_SCORE, CALL_SELECT, IKV_BF16, IKV_E2M1,  # noqa: F401
                  IKV_E4M3, IKV_F32, IKV_INT8, IKV_NO_XATTN, IKV_RESIDUAL, SYMBOLS, FreeSlots, IkvError, Pool,
                  QuantPool, Session, Sessions, Workspace, attend_chunk, attend_chunk_quant, decode_attend_quant,
                  decode_attend_slotmap, init_dead_slot, lib, make_free_slots, make_pool, make_quant_pool, qm_update,
                  quant_load, quant_store, quant_workspace_bytes, redirect_slots, return_slots, score_history,
                  select_budget, take_slots, timing, timing_read, workspace_bytes)
