"""MI355X-native batched token-ID BLEU (per-sentence and corpus) behind a C ABI.

The computation lives in `libtensorbleu.so` (hand-written HIP for gfx950, built from `csrc/` by
`python -m paper_2510_05485_amd.build`); `binding` marshals PyTorch device tensors into it.
`losses` holds what a training loop does with such rewards: losses over a policy's logits.  `embeddings`
is where a policy over token ids begins: rows of a table by ids, and their gradient.
"""
from .binding import (  # noqa: F401
    LIB_PATH, TB_DEV_LENGTH_RANGE, TB_DEV_TABLE_OVERFLOW, TB_DEV_TOKEN_RANGE, Stats, TensorBLEUError, allocate_workspace, load_library, make_config,
    tensorbleu_corpus, tensorbleu_count_clip, tensorbleu_dictionary, tensorbleu_finalize,
    tensorbleu_pack, tensorbleu_sentence, tensorbleu_status_string, tensorbleu_workspace_bytes,
    tensorbleu_workspace_layout, tensorrouge_n, tensorbleu_sentence_static,
    tensorbleu_static_scratch_bytes,
)
from .api import (  # noqa: F401
    BleuScorer, corpus_bleu, lengths_from_padding, pack_reference_lists, pad_references, rouge_n,
    sentence_bleu,
)
from .losses import (  # noqa: F401
    DistillationLoss, PolicyLoss, PreferenceLoss, TopLogprobs, distillation_loss, distillation_loss_grad,
    policy_loss, policy_loss_grad, preference_loss, preference_loss_grad, token_logprobs, top_logprobs,
)
from .embeddings import embedding, embedding_grad  # noqa: F401
