"""Quantised caches of the tests: storage of codes and scales as include/vxl.h states it, and inputs that reach its corners."""
import numpy as np
import torch

import oracle
from paper_2506_19225_amd import vxl, workloads as wl

FORMATS = ("fp4", "fp8")


def pack(codes, fmt):
    """uint8 codes [..., D] -> bytes [..., D * bits / 8]."""
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)) if fmt == "fp4" else codes


def quantised(k, v, fmt):
    """Oracle's (rows, scales) [Hkv, N, 2, ...] of k, v [Hkv, N, D], and the values they stand for."""
    (ck, sk), (cv, sv) = oracle.kvq_quantise(k, fmt), oracle.kvq_quantise(v, fmt)
    return (np.ascontiguousarray(np.stack([pack(ck, fmt), pack(cv, fmt)], 2)), np.ascontiguousarray(np.stack([sk, sv], 2)),
            oracle.kvq_values(ck, sk, fmt), oracle.kvq_values(cv, sv, fmt))


def device_cache(desc, fmt, rows, scales, spare=0):
    """A cache that holds these rows, and `spare` rows of NaN behind them."""
    rows = np.pad(rows, ((0, 0), (0, spare), (0, 0), (0, 0)), constant_values=0x77)
    scales = np.pad(scales, ((0, 0), (0, spare), (0, 0), (0, 0)), constant_values=255)
    return vxl.KvqCache(desc, fmt, rows=torch.from_numpy(rows).cuda(), scales=torch.from_numpy(scales).cuda())


def random_rows(rng, shape, dtype):
    """Values of very different magnitudes from row to row and block to block, as numpy float32 in storage precision."""
    x = rng.standard_normal(shape).astype(np.float32)
    x *= np.exp2(rng.integers(-6, 7, size=shape[:-1] + (1,))).astype(np.float32)
    x[..., : shape[-1] // 2] *= np.float32(0.37)
    return wl.round_to_bf16(x) if dtype == "bf16" else x
