"""One ALS half-sweep (the hot path of cuMF's alternating least squares) as hand-written
HIP kernels for the MI355X (gfx950), behind the C ABI of include/als.h.

``paper_1603_03820_amd.als`` is the ctypes binding (same names as the C entry points);
``paper_1603_03820_amd.driver`` runs whole iterations (update-X, update-Theta, RMSE) on top of it.
``paper_1603_03820_amd.serve`` answers with the factors they leave (include/als_serve.h): rows in 8 bits,
scores, and the draw of items; ``paper_1603_03820_amd.predict`` says how probable items are
(include/als_predict.h): predictions with offsets, log probabilities of items and their gradient.
"""
from .als import (ALS_F_MAX, ALSError, Context, als_csr_to_csc, als_destroy,  # noqa: F401
                  als_half_sweep, als_init, als_plan, als_rmse, als_rmse_waves, als_status,
                  als_workspace_bytes)

_LAZY = {}      # names whose library is not built: training does without it, and they say so
try:
    from .serve import (Recommender, als_quantize, als_sample, als_score,  # noqa: F401
                        als_serve_workspace_bytes)
except ImportError:
    _LAZY.update(dict.fromkeys(("serve", "Recommender", "als_quantize", "als_sample", "als_score",
                                "als_serve_workspace_bytes"), "serve"))
try:
    from .predict import (Predictor, als_log_prob, als_log_prob_grad, als_predict,  # noqa: F401
                          als_predict_workspace_bytes)
except ImportError:
    _LAZY.update(dict.fromkeys(("predict", "Predictor", "als_log_prob", "als_log_prob_grad", "als_predict",
                                "als_predict_workspace_bytes"), "predict"))


def __getattr__(name):
    if name not in _LAZY:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
    import importlib
    module = importlib.import_module("." + _LAZY[name], __name__)
    return module if name == _LAZY[name] else getattr(module, name)
