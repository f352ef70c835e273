"""One ALS half-sweep (the hot path of cuMF's alternating least squares) as hand-written
HIP kernels for the MI355X (gfx950), behind the C ABI of include/als.h.

``paper_1603_03820_amd.als`` is the ctypes binding (same names as the C entry points);
``paper_1603_03820_amd.driver`` runs whole iterations (update-X, update-Theta, RMSE) on top of it.
``paper_1603_03820_amd.serve`` answers with the factors they leave (include/als_serve.h): rows in 8 bits,
scores, and the draw of items.
"""
from .als import (ALS_F_MAX, ALSError, Context, als_csr_to_csc, als_destroy,  # noqa: F401
                  als_half_sweep, als_init, als_plan, als_rmse, als_rmse_waves, als_status,
                  als_workspace_bytes)

try:
    from .serve import (Recommender, als_quantize, als_sample, als_score,  # noqa: F401
                        als_serve_workspace_bytes)
except ImportError:      # libals_serve.so is not built: training does without it, and the serving names say so
    def __getattr__(name):
        if name not in ("serve", "Recommender", "als_quantize", "als_sample", "als_score", "als_serve_workspace_bytes"):
            raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
        import importlib
        serve = importlib.import_module(".serve", __name__)
        return serve if name == "serve" else getattr(serve, name)
