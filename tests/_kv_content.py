"""A cache of one sequence with given keys and values, for tests whose faults lie in the content."""
import numpy as np

import _decoder as R


def cache_of(rng, k, v, G, page=16):
    """R.Cache whose only sequence holds k, v [n][kv heads][D] (slots past its end: as R.Cache has them)."""
    n, Hkv, D = k.shape
    c = R.Cache(rng, 1, [n], Hkv, D, G, page)
    for name, x in (("k", k), ("v", v)):
        full = R.dequantize4(*getattr(c, name)).astype(np.float32)  # [pages][kv heads][page][D]
        for p in range(n):
            full[c.table[0, p // page], :, p % page] = x[p]
        setattr(c, name, R.quantize4(full, G))
    c.packed = [R.pack_codes(c.k[0], True), R.pack_params(*c.k[1:]), R.pack_codes(c.v[0], False),
                R.pack_params(*c.v[1:])]
    return c
