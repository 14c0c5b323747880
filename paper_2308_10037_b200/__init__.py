"""B200-native full-batch gradient-descent logistic regression (CUDA, sm_100a).

``datagen`` (seeded inputs) imports without the compiled library; the binding in ``api`` loads the
C-ABI shared library on first use and raises if it is missing -- there is no CPU fallback.
"""
_FROM_API = ("lr_loss_grad", "lr_fit", "lr_predict", "lr_embed", "lr_embed_grad", "lr_route", "lr_route_grad", "lr_ckpt8_save",
             "lr_ckpt8_load", "lr_ckpt8_grad", "lr_logp", "lr_logp_grad", "lr_policy_loss", "lr_pref_loss", "lr_distill_loss", "release_contexts", "Context", "LrError")
__all__ = ["datagen", "api", *_FROM_API]


def __getattr__(name):
    if name in _FROM_API:
        from . import api
        return getattr(api, name)
    raise AttributeError(name)
