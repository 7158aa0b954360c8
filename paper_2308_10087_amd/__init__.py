"""gnnstage: one pipeline stage of chunk-based pipelined GNN training on one MI355X.

The work is done by hand-written HIP kernels in ``libgnnstage.so`` (C ABI declared in
``include/gnnstage.h``); this package only marshals arguments.  There is no CPU fallback:
importing :mod:`binding` raises if the library has not been built.
"""
from .binding import (  # noqa: F401
    GNNSTAGE_BF16, GNNSTAGE_F32, GNNSTAGE_GCN, GNNSTAGE_GCNII, GNNSTAGE_RESGCN, GNNSTAGE_SAGE, GnnStage, GnnStageError, KIND_NAMES,
    gnnstage_dense_plan, gnnstage_plan_pack, gnnstage_plan_tasks, gnnstage_plan_transpose, gnnstage_version, lib,
    GNNTRAIN_ADAM, GNNTRAIN_SGD, GnnTrainer, gnntrain_adam_step, gnntrain_chunk_order, gnntrain_sgd_step,
    gnntrain_softmax_xent, gnntrain_sum, gnntrain_sum_static, gnnstage_partition_chunks, gnnstage_permute_csr,
    gnnstage_debug_gather_rate, gnntrain_head_xent, gnntrain_head_xent_workspace_size, gnnstage_rows8_load, gnnstage_rows8_store,
    GNNTRAIN_ADAMW, gnntrain_adamw_step, gnntrain_adamw_tensors, gnntrain_logprobs, gnntrain_logprobs_grad,
    gnntrain_logprobs_grad_workspace_size, gnntrain_logprobs_workspace_size,
    gnnstage_rows4_load, gnnstage_rows4_product, gnnstage_rows4_store, gnnstage_rows4_store_columns,
    gnnstage_rows8_weight_grad, gnnstage_rows8_weight_grad_workspace_size,
)
