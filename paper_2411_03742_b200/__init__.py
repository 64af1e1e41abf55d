"""AdaCons (arXiv 2411.03742) gradient aggregation for NVIDIA B200 (sm_100a).

The product is the C-ABI shared library built from `csrc/`; `AdaCons` in `binding`
marshals arguments to it.  There is no CPU fallback: using the class without the built
library raises.
"""
from . import workloads  # noqa: F401


_LAZY = {"AdaCons": "binding", "AdaConsError": "binding", "load_library": "binding", "Orthogonalizer": "orth",
         "attention_forward": "attention", "attention_backward": "attention", "Rope": "rope",
         "residual_norm_forward": "norms", "residual_norm_backward": "norms", "residual_norm": "norms",
         "feedforward_forward": "feedforward", "feedforward_backward": "feedforward", "gated_feedforward": "feedforward",
         "distill_forward": "distillation", "distill_backward": "distillation", "distill": "distillation"}


def __getattr__(name):
    if name in _LAZY or name in _LAZY.values():
        import importlib
        mod = importlib.import_module("." + _LAZY.get(name, name), __name__)
        if name not in _LAZY:
            return mod
        globals()[name] = value = getattr(mod, name)        # looked up once
        return value
    raise AttributeError(name)
