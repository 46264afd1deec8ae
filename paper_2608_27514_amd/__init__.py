"""MI355X (gfx950) trajectory-verification step for trajectory-level speculative
decoding of diffusion language models.

The three calls of one verification step (all HIP kernels in libtrajspec.so):

* :func:`verify_attn`      -- trajectory-masked attention over the dual cache and
  the packed draft blocks (each draft sees the cache, itself and its ancestors).
* :func:`confidence_topk`  -- per-position max-softmax confidence and top-k
  candidates over the vocabulary.
* :func:`accept`           -- threshold-decoding consistency and greedy /
  longest-path acceptance of the draft tree.

and the next step's drafts:

* :func:`build_tree`       -- confidence-stratified draft tree (Alg. 1) from the
  accepted state and the candidates its verification produced.

and inter-block speculation (Sec. 3.4):

* :func:`interblock_trigger` -- whether the next block is confident enough to
  speculate on both blocks; :func:`joint_peers` builds the visibility masks of the
  two blocks' joint trees on the device and :func:`verify_attn` with ``peers``
  verifies them in one pass.

and :func:`verify_layer`, a whole decoder layer of the verification forward pass around the
attention (norms, projections on the library's MFMA GEMM, RoPE, SwiGLU MLP), and
:func:`linear`, that GEMM on its own; :func:`refresh_layer` runs the same layer over whole
sequences at a block boundary and refreshes the dual cache (App. A).

For serving sequences of different lengths and requests with their own rules:

* :func:`paged_append` -- new tokens' keys rotated by position and written, with the values, into a
  paged key-value cache; :func:`paged_attn` attends to it.
* :func:`confidence_topk_adjusted` -- :func:`confidence_topk` under penalties for repeated tokens,
  biases and grammar masks.

and in 8 bits (e4m3 with a power-of-two scale per block), for steps that the cache's and the weights' bytes bound:

* :func:`paged_append8` and :func:`paged_attn8` -- the paged cache with a scale per block of tokens and head.
* :func:`quantize8` -- a weight matrix with a scale per block of 128 x 128, once; :func:`linear8` multiplies by it.
"""

from ._lib import (  # noqa: F401
    DEV_BAD_BLOCK,
    DEV_BAD_HISTORY,
    DEV_BAD_LENGTH,
    DEV_BAD_MASK,
    DEV_BAD_PAGE,
    DEV_BAD_ROOT,
    DEV_BAD_LEAF,
    DEV_BAD_PARENT,
    LIB_PATH,
    TrajSpecError,
    accept,
    build_tree,
    built_digest,
    check_build,
    confidence_topk,
    confidence_topk_adjusted,
    confidence_topk_adjusted_workspace_size,
    confidence_topk_noalloc,
    confidence_topk_workspace_size,
    device_status,
    interblock_trigger,
    joint_peers,
    layer_workspace_size,
    linear,
    linear8,
    linear8_workspace_size,
    linear_workspace_size,
    refresh_layer,
    refresh_layer_workspace_size,
    verify_layer,
    load,
    paged_append,
    paged_append8,
    paged_attn,
    paged_attn8,
    paged_attn8_workspace_size,
    paged_attn_workspace_size,
    quantize8,
    tree_max_nodes,
    verify_attn,
    verify_attn_workspace_size,
    version,
)
