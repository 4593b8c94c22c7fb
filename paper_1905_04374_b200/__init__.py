"""B200-native gradient aggregation rules (averaging, median, Krum, multi-Krum,
Bulyan, multi-Bulyan) behind the C ABI of include/gar.h, the operators a worker
runs before its gradient is aggregated (include/gar_worker.h), and a worker's layers (include/gar_linear.h).

`binding`, `worker` and `linear` marshal torch tensors into the C calls; `workloads` draws the seeded
synthetic inputs; `build` compiles libgar.so.  All arithmetic runs in the CUDA
kernels of csrc/.
"""
from . import workloads  # noqa: F401
from .binding import (  # noqa: F401
    DISTANCE_MODES, EVEN_MEDIAN, GAR_MAX_N, RULES, GarError, distance_path, gar_selftest_bounded_wait, GarParams, GarSelection, gar_aggregate, gar_aggregate_ex, gar_aggregate_host, gar_aggregate_multi, gar_multi_workspace_bytes, GarTensor, GarMultiParams,
    gar_beta, gar_coordinate_phase, gar_pairwise_distances, gar_pairwise_distances_static, gar_reduce_partials, gar_schedule_from_tables, gar_select, gar_shutdown,
    gar_last_cuda_error, gar_status_string, gar_theta, gar_version, gar_workspace_bytes, lib, new_selection, read_selection,
    write_selection,
)
from .worker import (  # noqa: F401
    ACTIVATIONS, GAR_MAX_TOP, Activation, ActivationGrad, Checkpoint, GarActivationGradParams, GarActivationParams, GarCheckpoint,
    GarLogprobsGradParams, GarLogprobsParams, GarWeightGradParams, TokenLogprobs, gar_activation_backward, gar_activation_forward,
    gar_checkpoint_pack, gar_checkpoint_unpack, gar_linear_weight_grad, gar_weight_grad_workspace_bytes, gar_token_logprobs, gar_token_logprobs_backward,
)
from .linear import (  # noqa: F401
    GarDropoutParams, GarGatedLinearGradParams, GarGatedLinearParams, GarLinearLogprobsGradParams, GarLinearLogprobsParams, GatedLinearGrad,
    LinearLogprobs, gar_dropout, gar_gated_linear_backward, gar_gated_linear_backward_workspace_bytes, gar_gated_linear_forward,
    gar_gated_linear_workspace_bytes, gar_linear_logprobs, gar_linear_logprobs_backward, gar_linear_logprobs_backward_workspace_bytes,
    gar_linear_logprobs_workspace_bytes,
)
