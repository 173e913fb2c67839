"""NOMAD Projection epoch path for AMD MI355X: a C-ABI HIP library (libnomad.so) and its binding.

Importing the package loads nothing; ``binding.load_library()`` opens the shared library and
raises if it has not been built."""
from .binding import (Nomad, NomadError, NomadConfig, load_library, knn_in_clusters, kmeans_lloyd, neighbourhood_preservation,
                      random_triplet_accuracy, random_triplet_accuracy_noalloc, pca_init, kmeans_lsh_init, release_memory, SCATTER_ATOMIC, SCATTER_DETERMINISTIC,
                      NOMAD_DEVICE, NOMAD_HOST, FAR_FIELD_EXACT, FAR_FIELD_SAMPLED, PATH_ATOMIC_FP32, PATH_BINNED,
                      PATH_BINNED_POOLED, PATH_FIXED_ATOMICS, PATH_NAMES, EDGES_ROWS, EDGES_RECORDS, EDGES_POOLED, EDGES_EXCHANGED, EDGES_LDS_SUMS, POOL_PICKS16, POOL_DISTINCT, POOL_STRATIFIED)  # noqa: F401

# the learned map's operators take torch's tensors, so their module brings torch with it: it is imported with the first of them
_OPERATORS = ("Routing", "State8", "adamw_state", "adamw_state_values", "adamw_step", "combine", "combine_gradient", "grouped_product",
              "grouped_weight_gradient", "route", "route_gradient")
__all__ = [name for name in globals() if not name.startswith("_")] + ["operators", *_OPERATORS]


def __getattr__(name):
    if name not in __all__:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
    import importlib
    operators = importlib.import_module(".operators", __name__)
    globals().update((each, getattr(operators, each)) for each in _OPERATORS)
    return globals()[name]


def __dir__():
    return sorted(set(globals()) | set(__all__))
