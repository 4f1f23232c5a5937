"""GB300-native joint evaluator (FlashEvaluator, arXiv 2603.02565).

The evaluation runs in libfe.so (hand-written sm_103a CUDA behind a C-ABI,
declared in include/fe.h); `binding.Evaluator` is its Python face, and
`generation` that of the candidate generator's operators (a paged cache with
shared-prefix attention, a policy loss).  Build the library with
`paper_2603_02565_gb300.build.build()`.
"""

__all__ = ["Evaluator", "FeError", "load_library"]
_GENERATION = ["PagedKV", "PolicyLoss", "check_status", "policy_loss", "policy_loss_backward", "rotary_table"]
__all__ += _GENERATION


def __getattr__(name):
    if name in _GENERATION:
        from . import generation
        value = globals()[name] = getattr(generation, name)  # found at once the next time
        return value
    if name in __all__:
        from . import binding
        return getattr(binding, name)
    raise AttributeError(name)
