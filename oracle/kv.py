"""Plain 64-bit implementation of the 4-bit key/value cache (test infrastructure only).

Everything is numpy on host copies, one sequence and head at a time, written from the format
and the formulas in include/oilbird.h.
"""
from __future__ import annotations

import numpy as np

GROUP = 64


def from16(bits: np.ndarray, dtype: str) -> np.ndarray:
    """16-bit patterns -> float64."""
    if dtype == "bf16":
        return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    return bits.view(np.float16).astype(np.float64)


def to16(x: np.ndarray, dtype: str) -> np.ndarray:
    """float64 -> 16-bit patterns, one rounding to nearest even (finite inputs)."""
    if dtype == "f16":
        return x.astype(np.float16).view(np.uint16)
    # float64 -> 8 significant bits directly: scale to an integer significand and round
    out = np.zeros(x.shape, np.float64)
    nz = x != 0
    e = np.maximum(np.floor(np.log2(np.abs(x[nz]))), -126) - 7
    out[nz] = np.rint(x[nz] / 2.0 ** e) * 2.0 ** e
    return (out.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


def channel_bit() -> np.ndarray:
    """First bit of each channel's code in the 256 bits of a group."""
    ch = np.arange(GROUP)
    return 32 * (ch // 8) + 4 * (ch % 8 // 2) + 16 * (ch % 2)


def decode_block(block: np.ndarray, page: int, head_dim: int, dtype: str):
    """Bytes of one (page, head) block -> dict with k, v [page, head_dim] float64 and the codes and
    meta they come from."""
    groups = head_dim // GROUP
    part = groups * page * 36
    bit = channel_bit()
    out = {}
    for name, b in (("k", block[:part]), ("v", block[part:2 * part])):
        raw = b[: groups * page * 32].reshape(groups, page, 32)
        code = raw[:, :, bit // 8] >> (bit % 8) & 15                       # [groups, page, 64]
        meta = b[groups * page * 32:].copy().view(np.uint16).reshape(page, groups, 2)
        scale, low = from16(meta[..., 0], dtype), from16(meta[..., 1], dtype)
        with np.errstate(invalid="ignore"):
            x = scale[..., None] * code.transpose(1, 0, 2) + low[..., None]
        out[name] = x.reshape(page, head_dim)
        out[name + "_code"] = code.transpose(1, 0, 2).reshape(page, head_dim)
        out[name + "_scale"], out[name + "_low"] = meta[..., 0], meta[..., 1]
    return out


def gather(pages: np.ndarray, table: np.ndarray, length: int, head: int, page: int, head_dim: int,
           dtype: str):
    """k, v [length, head_dim] and has [length] (False: the slot's page is none) of one sequence;
    pages: [n_pages, n_kv, block bytes]."""
    k, v = np.zeros((length, head_dim)), np.zeros((length, head_dim))
    has = np.zeros(length, bool)
    for p0 in range(0, length, page):
        p, n = int(table[p0 // page]), min(page, length - p0)
        if 0 <= p < pages.shape[0]:
            d = decode_block(pages[p, head], page, head_dim, dtype)
            k[p0:p0 + n], v[p0:p0 + n], has[p0:p0 + n] = d["k"][:n], d["v"][:n], True
    return k, v, has


def quantise(x: np.ndarray, dtype: str):
    """[..., 64] float64 of 16-bit elements -> codes, scale, low (exact arithmetic up to float64)."""
    low, high = x.min(-1), x.max(-1)
    scale = from16(to16((high - low) / 15, dtype), dtype)
    with np.errstate(divide="ignore", invalid="ignore"):
        code = np.clip(np.rint((x - low[..., None]) / scale[..., None]), 0, 15)
    return np.where(scale[..., None] > 0, code, 0), scale, low


def attend(q, k, v, sees, scale):
    """q [rows, d]; k, v [slots, d]; sees [rows, slots] -> out [rows, d], lse [rows]."""
    s = np.where(sees, (q @ k.T) * scale, -np.inf)
    top = s.max(-1, initial=-np.inf)
    with np.errstate(invalid="ignore", divide="ignore"):
        p = np.exp(s - np.where(np.isfinite(top), top, 0)[:, None])
        total = p.sum(-1)
        out = np.where(total[:, None] == 0, 0.0, (p @ np.where(sees.any(0)[:, None], v, 0)) / total[:, None])
        lse = np.where(total == 0, -np.inf, np.log(total) + np.where(np.isfinite(top), top, 0))
    return out, lse


def evict(weight, pos, n_pos, budget, sink, recent):
    """Slots of one (sequence, head) -> source slot of each of the first `budget` slots."""
    n = len(weight)
    w = np.where(np.isnan(weight), -np.inf, weight).astype(np.float64)
    safe = (pos < sink) | (pos >= n_pos - recent)
    order = sorted(range(n), key=lambda i: (not safe[i], 0.0 if safe[i] else -w[i], pos[i], i))
    keep = np.zeros(n, bool)
    keep[order[:budget]] = True
    src = np.arange(min(n, budget))
    holes, movers = np.nonzero(~keep[:budget])[0], budget + np.nonzero(keep[budget:])[0]
    src[holes] = movers
    return src
