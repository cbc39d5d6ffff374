"""MI355X-native learned-optimizer step (small_fc_lopt, VeLO) and the operators of the training loop around it (`ops`:
token log probabilities, layer norm, dropout, KL divergence, policy and preference losses, gradient clipping): thin binding over liblopt.so.

Every step of the optimizer and every operator runs in the HIP kernels behind the C boundary of include/lopt.h;
this package only marshals arguments. There is no CPU fallback: if the library is not built,
loading it raises.
"""
from .binding import (LoptError, LearnedOptimizer, lib, lopt_config, lopt_tensor_desc,  # noqa: F401
                      default_config, weights_count, LOPT_SMALL_FC, LOPT_VELO)


def __getattr__(name):
    # the torch.optim veneer and the operators import torch at module level; load them on first use only
    if name == "ops":
        import importlib
        return importlib.import_module(".ops", __name__)
    if name == "LearnedOptTorch":
        from .optim import LearnedOptTorch
        return LearnedOptTorch
    raise AttributeError(name)
