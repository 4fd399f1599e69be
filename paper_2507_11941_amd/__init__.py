"""MI355X-native byte-level BPE batch encoder (BlockBPE's hot path), and operators on the token batches it writes.

Thin Python binding over the C ABI in ``include/bpe.h`` and ``include/bpe_ops.h`` (``libbpe_hip.so``, hand-written HIP for
gfx950).  PyTorch is used for device memory and streams only; every step runs in the library's kernels.
There is no CPU fallback: if the library is missing or no GPU is present the calls raise.
"""
from ._binding import (BpeError, Table, build_table, build_table_vocab, encode_batch, encode_batch_static, encode_strings, read_profile, lib_path, load_library,
                       set_profiling, table_image, workspace_bytes, MAX_STRING_BYTES)
from ._ops import (embed_tokens, embed_tokens_grad, next_tokens, policy_loss, preference_loss, token_logprobs,
                   token_logprobs_and_grad, token_logprobs_grad)

__all__ = ["BpeError", "Table", "build_table", "build_table_vocab", "encode_batch", "encode_batch_static", "encode_strings", "read_profile", "lib_path",
           "load_library", "set_profiling", "table_image", "workspace_bytes", "MAX_STRING_BYTES",
           "embed_tokens", "embed_tokens_grad", "next_tokens", "policy_loss", "preference_loss", "token_logprobs",
           "token_logprobs_and_grad", "token_logprobs_grad"]
