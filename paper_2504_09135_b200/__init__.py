"""B200 (sm_100a) implementation of the DISC + PPV constrained-decoding hot path.

The work is done by the CUDA library built from csrc/ (C ABI: include/disc.h); this package is
its Python binding plus a small decode-loop helper.  Nothing here falls back to the CPU.
"""
from .binding import (DISC_BF16, DISC_F16, DISC_F32, ROW_DEAD, ROW_DONE, ROW_NOMASS, ROW_NONFINITE, ROW_NOPAGE, DiscError,
                      DiscSet, DiscState, StepOutputs, disc_accept, disc_accept_resample, disc_build_set, disc_build_set_eok, disc_mask,
                      disc_mask_static, disc_project_check, disc_project_scratch, disc_project_step, disc_resample, disc_sampling_uniforms, disc_set_rows, disc_state_init, disc_step, disc_step_topm, disc_topm, disc_verify,
                      lib)
from .decoder import DiscDecoder
from .model_ops import (AttendPlan, DiscCache, disc_attend_cached, disc_attend_check, disc_attend_plan, disc_attend_prompt,
                        disc_cache_compact, disc_cache_extend, disc_cache_fork, disc_cache_free, disc_cache_read, disc_cache_write,
                        disc_logprobs, disc_logprobs_grad, disc_norm_rope, disc_norm_rope_grad, disc_norm_rope_write)

__all__ = ["DISC_BF16", "DISC_F16", "DISC_F32", "ROW_DEAD", "ROW_DONE", "ROW_NOMASS", "ROW_NONFINITE", "ROW_NOPAGE", "DiscError",
           "DiscSet", "DiscState", "StepOutputs", "disc_accept", "disc_accept_resample", "disc_build_set", "disc_build_set_eok", "disc_mask",
           "disc_mask_static", "disc_project_check", "disc_project_scratch", "disc_project_step", "disc_resample", "disc_sampling_uniforms", "disc_set_rows", "disc_state_init", "disc_step", "disc_step_topm", "disc_topm", "disc_verify",
           "AttendPlan", "DiscCache", "disc_attend_cached", "disc_attend_check", "disc_attend_plan", "disc_attend_prompt",
           "disc_cache_compact", "disc_cache_extend", "disc_cache_fork", "disc_cache_free", "disc_cache_read", "disc_cache_write",
           "disc_logprobs", "disc_logprobs_grad", "disc_norm_rope", "disc_norm_rope_grad", "disc_norm_rope_write",
           "lib", "DiscDecoder"]
