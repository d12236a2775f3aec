"""R-FAST activation rounds on MI355X: thin ctypes binding over librfast.so.

Nothing here computes: every step of the round runs in the HIP kernels.  The
library must have been built (python -m paper_2307_11617_amd.build); loading
fails loudly otherwise."""
from .binding import (RFAST_FIELDS, RFast, RFastError, RfastProblem, lib, rfast_check, rfast_common_roots, rfast_create,  # noqa: F401
                      rfast_destroy, rfast_diagnostics, rfast_diagnostics_static, rfast_init, rfast_kernel_time, rfast_last_error,
                      rfast_profile_enable, rfast_read_state, rfast_rebase, rfast_set_rebase_interval, rfast_set_optimizer, rfast_set_gamma_schedule, rfast_sync_round, rfast_sync_run, rfast_round, rfast_run, rfast_run_generated, rfast_run_events, rfast_use_graphs, rfast_use_blocks, rfast_block_info, rfast_set_tile_group, rfast_set_wait_limits, rfast_workspace_bytes,
                      rfast_write_state, rfast_adamw_state_bytes, rfast_set_adamw)
from .operators import (RFastAdamW, RFastRoute, rfast_adamw_create, rfast_adamw_destroy, rfast_adamw_set_steps, rfast_adamw_step,  # noqa: F401
                        rfast_adamw_steps, rfast_adamw_workspace_bytes, rfast_lora_backward, rfast_lora_forward,
                        rfast_lora_workspace_bytes, rfast_softmax_xent, rfast_policy_loss, rfast_embedding, rfast_embedding_backward,
                        rfast_embedding_backward_workspace_bytes, rfast_route, rfast_route_plan, rfast_route_backward, rfast_route_gather,
                        rfast_route_combine, rfast_route_combine_backward, rfast_route_workspace_bytes)
