"""MI355X (gfx950) commit step of Reliable Parallel Decoding.

``binding`` wraps the C ABI of ``librpd.so`` (include/rpd.h); ``workload``
draws seeded synthetic inputs of the paper's model shapes."""
from .binding import (Params, QuantHead, RpdError, ScoreCommit, VerifyDraft, abi_version, distill,  # noqa: F401
                      distill_grad, gate_commit, last_error, lib, score_commit, status_string, verify_draft,
                      workspace_size)
