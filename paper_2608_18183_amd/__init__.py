"""MI355X (gfx950) batched speculative-Jacobi rollout (HB-SJD).

Python binding of the C ABI in include/hbsjd.h: argument marshalling only;
every step of the rollout runs in the HIP library libhbsjd.so. PyTorch supplies
device memory and the stream. Importing this package does not load the
library; the first call does, and raises if it has not been built.
"""
from .binding import (  # noqa: F401
    DTYPE_BF16, DTYPE_F32, ELEM_BF16, ELEM_F16, ELEM_F32, KERNELS, EXEC_AUTO, EXEC_COMPACT, EXEC_FULL, VERIFY_AR, VERIFY_AR_GREEDY,
    VERIFY_GREEDY, VERIFY_PROB, PROGRESS_INDEPENDENT, PROGRESS_SYNC,
    HbsjdError, Context, ModelDesc, hbsjd_adjust_rows, hbsjd_bikl_rows, hbsjd_distill_top_rows,
    hbsjd_mfma_probe, hbsjd_philox, hbsjd_top_logits_rows, hbsjd_transform_rows,
    hbsjd_verify_probs,
    hbsjd_version,
    library_path, load_library,
)
