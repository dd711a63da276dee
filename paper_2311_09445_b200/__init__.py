"""B200-native Prioritized Replay Buffer (the Replay Manager + Data Storage of PEARL,
arXiv 2311.09445): a K-ary sum tree over transition priorities with batched insert,
stratified prefix-sum sampling, importance-sampling weights, gather and priority update,
as hand-written CUDA behind a C ABI.  `PrioritizedReplay` is the thin Python binding.
Beside it `RowRouter`: rows of a batch chosen, weighed and moved (expert layers with their
gradients, beam search), and `RowLayers`, which has a layer's operators too (norm, dropout, a
whole expert layer for a few rows)."""
from .binding import PearlError, PrioritizedReplay, load_library  # noqa: F401
from .layers import RowLayers  # noqa: F401
from .routing import RowRouter  # noqa: F401

__all__ = ["PrioritizedReplay", "RowRouter", "RowLayers", "PearlError", "load_library"]
