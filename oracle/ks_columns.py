"""fp64 oracle of the learned columns (test infrastructure, like ``ks_oracle``; no code
shared with the HIP library): the draws of dropout, the lookup of a table's rows, the
table's gradient and bounds on what fp32 arithmetic may be off.  The loss at given z
is ``ks_fit.eta_loss``, family by family."""
from __future__ import annotations

import numpy as np

EPS = 2.0 ** -24          # half a step of fp32, relative
HALF = {"f32": EPS, "bf16": 2.0 ** -8}
M32 = (1 << 32) - 1


def philox(counter, key):
    """Philox4x32-10 (Salmon et al. 2011) of one counter (four words) and key (two)."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & M32, (a >> 32) ^ c[3] ^ k[1], a & M32]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    return c


def philox_many(block, step, site, seed):
    """The words [n][4] of blocks [n]."""
    u = np.uint64
    block = np.asarray(block, u)
    c = [block & u(M32), block >> u(32), np.full(block.shape, step, u), np.full(block.shape, site, u)]
    k0, k1 = seed & M32, seed >> 32
    for _ in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> u(32)) ^ c[1] ^ u(k0), b & u(M32), (a >> u(32)) ^ c[3] ^ u(k1), a & u(M32)]
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    return np.stack(c, -1).astype(np.uint32)


def least(p):
    return int(np.floor(p * 65536 + 0.5))


def keep(rows, cols, p, seed, site=0, step=0):
    """[len(rows)][cols]: whether the elements of these rows stay, and what they are then
    multiplied by."""
    per = -(-cols // 8)
    block = np.asarray(rows, np.uint64)[:, None] * np.uint64(per) + np.arange(per, dtype=np.uint64)
    words = philox_many(block, step, site, seed)
    draws = np.stack([words & 0xFFFF, words >> 16], -1).reshape(len(rows), 8 * per)[:, :cols]
    t = least(p)
    return draws >= t, 65536.0 / (65536 - t) if t < 65536 else 0.0


def drop(x, p, seed, site=0, step=0):
    k, up = keep(np.arange(x.shape[0]), x.shape[1], p, seed, site, step)
    return np.where(k, np.where(k, x, 0.0) * up, 0.0)


def embed(table, scale, ids, dropout=None):
    """dropout: the arguments of ``drop`` behind x, or None."""
    ids = np.asarray(ids, np.int64) & M32
    known = ids < table.shape[0]
    y = np.where(known[:, None], table[np.where(known, ids, 0)] * scale, 0.0) if len(table) else np.zeros((len(ids), table.shape[1]))
    return y if dropout is None else drop(y, *dropout)


def order(ids, n_ids):
    """row, id and off of ks_id_order."""
    key = np.minimum(np.asarray(ids, np.int64) & M32, n_ids)
    row = np.argsort(key, kind="stable")
    return row, key[row], np.searchsorted(key[row], np.arange(n_ids + 1))


def embed_back(ids, n_ids, dy, scale, dropout=None):
    """The table's gradient and a bound on its error in fp32: the additions that one
    term goes through, at most those of an id's rows; a longer sum goes by 64 in a row,
    then at most 64 such, then at most 9 joinings, all beyond in 64 bits.  scale times
    1 / (1 - p) is rounded once, its product with the sum once, the sum from 64 bits once."""
    row, _, off = order(ids, n_ids)
    d = np.asarray(dy, np.float64)
    d = (d if dropout is None else drop(d, *dropout))[row]
    # (rows without an id, at the end, belong to none)
    ends = off[:-1], off[1:]
    def sums(v):
        c = np.concatenate([np.zeros((1, v.shape[1])), np.cumsum(v, 0, dtype=np.longdouble)])
        return np.asarray(c[ends[1]] - c[ends[0]], np.float64)
    count = (ends[1] - ends[0])[:, None]
    big = sums(np.abs(d)) * abs(scale)
    return sums(d) * scale, (np.minimum(count, 64 + 64 + 9) + 3) * EPS * big


def eta_bounds(z, eta, weight, huber, loss, dz):
    """Bounds on the fp32 errors of one family's loss and dz (``ks_fit.eta_loss``): log(1 +
    e^-z) and log eta are within 8 half steps of their sizes, sigma(-z) and each of the
    products likewise; a sigma(-z) or a product below fp32's normal range (2^-126: z above 87)
    may be 0."""
    from oracle import ks_fit
    w = ks_fit.counted(eta, weight)
    on = w > 0
    if not on.any():
        return 0.0, np.zeros(len(w))
    z = np.where(on, z, 0.0)
    log_eta = np.log(np.where(on, eta, 1.0))
    size = np.logaddexp(0, -z) + np.abs(log_eta)
    er = 8 * EPS * (size + np.minimum(1, np.exp(-np.abs(z))))
    res = np.abs(np.logaddexp(0, -z) - log_eta)
    share = w / w.sum()
    slope = np.minimum(res + er, huber)
    bound = (share * (slope * er + 8 * EPS * slope * (res + er))).sum() + 4 * EPS * loss
    tiny = 2.0 ** -126
    return bound, share * (er * ks_fit.sigmoid(-z) + slope * (8 * EPS * ks_fit.sigmoid(-z) + tiny)) + 8 * EPS * np.abs(dz) + 3 * tiny
