"""1-bit Adam's compression-stage hot path on AMD MI355X (gfx950).

The kernels and their C ABI live in ``libonebit.so`` (sources in ``csrc/``,
header ``include/onebit.h``); this package is the Python binding.
"""
from .onebit import (  # noqa: F401
    Plan, State, SERVER_TABLES_AUTO, SERVER_TABLES_OFF, SERVER_TABLES_ON, onebit_decode, onebit_decompress_update, onebit_error_materialize,
    onebit_plan_create,
    onebit_server_reduce_compress, onebit_step, onebit_step_noalloc, onebit_warmup_adam_step,
    onebit_worker_compress, onebit_uncompressed_step, onebit_adam_message_step, onebit_l1_norm,
)
from .attention import (  # noqa: F401
    attention_workspace, onebit_attention_forward, onebit_attention_grad,
)
from .embedding import (  # noqa: F401
    embedding_workspace, onebit_embedding_forward, onebit_embedding_grad,
)
from .freeze import VarianceFreezeDetector  # noqa: F401
from .loss import (  # noqa: F401
    onebit_distill_forward, onebit_distill_grad, onebit_logprobs_forward, onebit_logprobs_grad,
)
from .muon import (  # noqa: F401
    Matrices, Muon, MUON_SCALE_NONE, MUON_SCALE_RMS, MUON_SCALE_SPECTRAL, PRODUCTS_F16,
    PRODUCTS_F32, matrices_kernels, onebit_muon_step, onebit_orthogonalize, products_for,
)
from .norm import (  # noqa: F401
    layer_norm_workspace, onebit_layer_norm_forward, onebit_layer_norm_grad,
)
from .optimizer import OnebitAdam  # noqa: F401
from ._native import OnebitError, lib  # noqa: F401
