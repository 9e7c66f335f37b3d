"""MI355X-native PAG (Projection-Augmented Graph) search: thin Python binding over the C ABI.

    from paper_2603_06660_amd import PagIndex
    ix = PagIndex.build(base_cuda, metric="ip", max_degree=32, num_subspaces=32, ef_construction=100)
    ids, dists = ix.search(queries_cuda, K=10, efS=64)

    from paper_2603_06660_amd import KvCache, KvTables      # keys and values in 8 bits, attention over them and over search results
    step = tables.extend(add, total); cache.append(k, v, step.slots)
    out, lse = cache.attend_selected(q, ids.view(tokens, heads, K), step, window=64)

All computation runs in libpag_hip.so (hand-written HIP kernels for gfx950); torch only
provides device memory and the stream.  Importing this package does not load the library;
the first use does, and raises if it has not been built.
"""
from .binding import (PagIndex, PagError, load_library, library_path, EXPORTED_SYMBOLS,  # noqa: F401
                      L2, IP, COS, FLAG_NO_PRT, FLAG_NO_PES, FLAG_FP16_VECTORS, FLAG_KEEP_ORDER,
                      FLAG_EXACT_TEST_COUNT, FLAG_PERMUTATION_TRANSFORM, FLAG_KEEP_QUERY_ORDER)


def __getattr__(name):      # these need torch, which importing the package does not
    if name in ("KvCache", "KvStep", "KvTables"):
        from . import kv
        return getattr(kv, name)
    raise AttributeError("module %r has no attribute %r" % (__name__, name))
