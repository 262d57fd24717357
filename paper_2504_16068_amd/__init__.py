"""MI355X-native Allegro channel-wise tensor product (arxiv 2504.16068, §II.D).

The compute lives in liballegro_tp.so (hand-written HIP for gfx950 behind the
C ABI of include/allegro_tp.h and include/allegro_layer.h) and in
liballegro_latent.so (the operators of the latent track,
include/allegro_latent.h); this package is their build scripts and a thin ctypes
binding with the same entry-point names.  Importing the package raises if
liballegro_tp.so has not been built, and using a name of the latent track if
liballegro_latent.so has not been: there is no CPU fallback.
"""

import os as _os

from .binding import (  # noqa: F401
    ALLEGRO_DETERMINISTIC,
    ALLEGRO_E_HIP,
    ALLEGRO_E_INVALID,
    ALLEGRO_E_NOMEM,
    ALLEGRO_E_TIMEOUT,
    ALLEGRO_E_UNSUPPORTED,
    ALLEGRO_FULL_PARITY,
    ALLEGRO_OK,
    ALLEGRO_VALIDATE,
    AllegroError,
    Plan,
    allegro_env_embed,
    allegro_last_error,
    allegro_layer_backward,
    allegro_layer_buffers,
    allegro_layer_forward,
    allegro_sh_backward,
    allegro_sh_forward,
    allegro_tp_backward,
    allegro_tp_backward_train,
    allegro_tp_backward_train_noalloc,
    allegro_tp_backward_workspace,
    allegro_tp_forward,
    allegro_tp_plan_create,
    allegro_tp_plan_destroy,
    layer_weight_shapes,
)
_LATENT = (
    "latent",
    "ALLEGRO_ACT_NONE",
    "ALLEGRO_ACT_SILU",
    "ALLEGRO_BF16",
    "ALLEGRO_F32",
    "allegro_group_rows",
    "allegro_group_rows_workspace",
    "allegro_grouped_matmul",
    "allegro_grouped_matmul_backward",
    "allegro_grouped_matmul_fp8",
    "allegro_grouped_matmul_workspace",
    "allegro_latent_last_error",
    "allegro_rms_norm_backward",
    "allegro_rms_norm_forward",
    "allegro_rms_norm_fp8",
    "allegro_rms_norm_workspace",
)


def __getattr__(name):
    """Names of the latent track, whose library need not be there for the rest of the package."""
    if name not in _LATENT:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
    import importlib

    module = importlib.import_module(".latent", __name__)
    globals().update({n: getattr(module, n) for n in _LATENT if n != "latent"})
    return globals()[name]


if _os.path.exists(_os.path.join(_os.path.dirname(_os.path.abspath(__file__)), "liballegro_latent.so")):
    __getattr__("latent")
