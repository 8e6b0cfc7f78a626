"""Fused sparse attention (3S) on AMD MI355X: Python side of libf3s.so.

    import paper_2505_08098_amd as f3s
    plan = f3s.Plan(row_ptr, col_idx, N)          # device int32 CSR
    O = f3s.run(plan, Q, K, V, scale=1/d**0.5)    # fp16 in, fp32 out

and dense attention for decoders (see ``dense``): ``CrossPlan``, ``cross_forward``,
``cross_backward`` over an encoder's states; ``WindowPlan``, ``window_forward``,
``window_backward``: causal, with a sliding window and sinks; ``Cache``,
``cache_write``, ``cache_read``, ``cache_keep``, ``cache_attend``, ``cache_attend_window``,
``cache_attend_tree`` over an 8-bit key/value cache; ``PagePool``, ``pages_assign``: its pages.

The compute path is the HIP library only (see ``binding``); ``workloads``
holds the seeded synthetic inputs.
"""
from .binding import (F3SError, Plan, PlanInfo, backward, forward,  # noqa: F401
                      forward_typed, load_library, probe_gather, probe_rows, probe_stream,
                      run, run_raw, run_trace, status_string, wall_clock_khz)
from .dense import (Cache, CrossPlan, PagePool, WindowPlan, cache_attend,  # noqa: F401
                    cache_attend_tree, cache_attend_window, cache_keep, cache_read,
                    cache_write, cross_backward, cross_forward, pages_assign,
                    window_backward, window_forward)
