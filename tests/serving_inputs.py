"""Inputs of the serving operators' GPU tests: paged caches with ragged lengths
on shuffled pages, whatever no request owns poisoned with NaN."""
import numpy as np

PS = 16


def bf16_bits(x):
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((u + 0x7fff + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def to_dev(a):
    import torch
    a = np.ascontiguousarray(a)
    t = torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a)
    return (t.view(torch.bfloat16) if a.dtype == np.uint16 else t).cuda()


def back(t):
    import torch
    t = t.cpu()
    return t.view(torch.int16).numpy().view(np.uint16) if t.dtype == torch.bfloat16 else t.numpy()


def typed(x, dtype):
    return bf16_bits(x) if dtype == "bf16" else np.ascontiguousarray(x, np.float32)


class Cache:
    """Pools with `reach[r]` places owned by request r, the first `filled[r]` of them holding values."""

    def __init__(self, rng, filled, hkv, d, dtype, reach=None, spare_columns=1, scale=1.0):
        filled = np.asarray(filled, np.int64)
        reach = filled if reach is None else np.asarray(reach, np.int64)
        pages = -(-reach // PS)
        self.pages = int(pages.sum()) + 3
        perm = rng.permutation(self.pages)
        self.table = np.full((len(filled), int(pages.max(initial=0)) + spare_columns), -1, np.int32)
        k = np.full((self.pages, hkv, PS, d), np.nan, np.float32)
        v = k.copy()
        at = 0
        for r, n in enumerate(pages):
            mine = perm[at:at + n]
            at += n
            self.table[r, :n] = mine
            for e, p in enumerate(mine):
                m = int(min(PS, max(0, filled[r] - e * PS)))
                k[p, :, :m] = rng.standard_normal((hkv, m, d)) * scale
                v[p, :, :m] = rng.standard_normal((hkv, m, d))
        self.k, self.v = typed(k, dtype), typed(v, dtype)


def attention_bound(dtype, out, size, reach, keys, d):
    """How far a result may be from fp64's `out`, from the roundings on the way.
    bf16: the weights are rounded (half a step, 2^-8) in the numerator and the
    denominator alike, and so is the output; scores and exponentials in fp32
    move a weight by less than 2^-14.  fp32: a dot product of d terms within
    d half steps of the sum of their magnitudes (<= reach), sums over the keys
    within `keys` half steps, 32 for the exponential and the rest."""
    if dtype == "bf16":
        return 2.0 ** -8 * (size + 2 * np.abs(out)) + 2.0 ** -14 * size + 1e-30
    return 2.0 ** -24 * (2 * (d + 2) * reach + keys + 32) * 2 * size + 1e-30
