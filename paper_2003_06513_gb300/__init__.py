"""Pattern-pruned 3x3 convolution on one GB300 (arXiv 2003.06513): inference, pruning and retraining.

The C library (``include/patconv.h``, built in-tree by ``build.py``) holds the whole path: the
host packer (pattern projection §4.3, connectivity pruning §4.4, filter grouping and compact
storage §3.4) and the sm_103a CUDA kernels (pattern-sparse convolution with fused bias + ReLU,
depthwise variant, max-pool), and the operators of masked retraining (``norm``: group norm with its
activation, forward and backward; ``optim``: gradient norm and AdamW over many tensors), which
``retrain`` runs together.  This package is a thin binding over it; ``workloads`` holds the seeded
synthetic inputs.  Importing the package does not load the library; the first call that needs it does,
and fails loudly if it cannot be built or loaded.
"""

__all__ = ["Layer", "pp_pack", "pp_conv", "pp_maxpool2x2", "default_patterns", "group_norm", "pp_group_norm",
           "pp_group_norm_backward", "AdamW", "GradNorm", "taps_of", "Retrainer", "PatconvError"]


def __getattr__(name):
    if name in ("Layer", "pp_pack", "pp_conv", "pp_maxpool2x2", "default_patterns"):
        from . import api
        return getattr(api, name)
    if name in ("group_norm", "pp_group_norm", "pp_group_norm_backward"):
        from . import norm
        return getattr(norm, name)
    if name in ("AdamW", "GradNorm", "taps_of"):
        from . import optim
        return getattr(optim, name)
    if name == "Retrainer":
        from . import retrain
        return retrain.Retrainer
    if name == "PatconvError":
        from ._lib import PatconvError
        return PatconvError
    raise AttributeError(name)
