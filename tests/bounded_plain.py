"""Attention with a sliding window and sinks, attention weights and eviction, in 64 bits and from the definitions in include/mpfa.h (test
helper; numpy only, on what the library's buffers hold).

The operands are what the quantizers left, so nothing here is rounded but P.  attend() also says how far an output may be from a
computation of the same in FP32 (derivation there)."""
import numpy as np

from layouts import codes_to_logical, paged_delta_to_logical, paged_k_to_logical, paged_v_to_logical, sf_to_logical

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6])
_e = np.arange(256)
E4M3 = np.where((_e >> 3 & 15) == 0, (_e & 7) * 2.0 ** -9, 2.0 ** ((_e >> 3 & 15) - 7.0) * (1 + (_e & 7) / 8)) * np.where(_e >= 128, -1.0, 1.0)
E4M3[[127, 255]] = np.nan

# The exponent lam (S - m) is up to some 64 in magnitude and made of four FP32 operations (the tensor core's three additions of S, the
# product, the subtraction): off by at most 4 x 64 x 2^-24 = 2^-16, so P by 2^-16 ln 2 relative and 2 units of 2^-23 of the hardware's 2^x.
NEAR = 2.0 ** -15
# Sums of up to some thousand terms in FP32, on a tensor core that drops what lies behind the accumulator's last bit: 2^-23 of the
# accumulator for each addition of a block's 4 MMAs, some 2^7 of them; the factors between blocks and l: as NEAR.
SUMS = 2.0 ** -15


def e2m1(codes):
    return E2M1[np.stack((codes & 15, codes >> 4), -1)].reshape(*codes.shape[:-1], -1)


def tile_rows(t):
    """Fp4Tensor -> [B, H, N, 128]"""
    c, _ = codes_to_logical(t.codes.cpu().numpy(), t.B, t.H, t.N)
    s = sf_to_logical(t.sf.cpu().numpy(), t.B, t.H, t.N)[:, :, :t.N]
    return e2m1(c) * np.repeat(E4M3[s], 16, -1)


def bf16(t):
    return t.float().cpu().numpy().astype(np.float64)


def cached(kv, table_row, L, pages=None):
    """Tokens 0..L-1 of one request: K [H_kv, L, 128], V, Delta_S [H_q, L]; pages: logical pages that exist (the others: zeros)."""
    n = -(-L // 64)
    G = kv.H_q // kv.H_kv
    K, V = np.zeros((kv.H_kv, n * 64, 128)), np.zeros((kv.H_kv, n * 64, 128))
    D = np.zeros((kv.H_q, n * 64))
    for i in range(n) if pages is None else pages:
        p = int(table_row[i])
        k = e2m1(paged_k_to_logical(kv.k_codes[p].cpu().numpy()))
        s = E4M3[kv.k_sf[p].cpu().numpy().reshape(kv.H_kv, 64, 8)]
        K[:, i * 64:i * 64 + 64] = k * np.repeat(s, 16, -1)
        V[:, i * 64:i * 64 + 64] = E4M3[paged_v_to_logical(kv.v_fp8[p].cpu().numpy())]
        if kv.delta is not None:
            D[:, i * 64:i * 64 + 64] = paged_delta_to_logical(bf16(kv.delta[p]), G)
    return K[:, :L], V[:, :L], D[:, :L]


def visible(pos, n_kv, window, sinks):
    """[rows, keys]"""
    j, p = np.arange(n_kv)[None], np.asarray(pos)[:, None]
    return (j <= p) & ((j > p - window) | (j < sinks))


def lists_of_blocks(see, part):
    """The 128-key blocks with a key that some row sees, ascending, in runs of `part` (0: one run)."""
    blocks = [u for u in range(-(-see.shape[1] // 128)) if see[:, u * 128:u * 128 + 128].any()]
    return [blocks] if not part else [blocks[i:i + part] for i in range(0, len(blocks), part)]


def p_hat(x):
    """E4M3(x), 0 <= x <= 448, and the distance to the code's neighbour across the nearer border where x is within NEAR of it, else 0."""
    step = np.exp2(np.floor(np.log2(np.maximum(x, 2.0 ** -6))) - 3)
    q = np.round(x / step)
    border = np.abs(x / step - np.floor(x / step) - 0.5) * step <= NEAR * x
    return q * step, np.where(border, step, 0.0)


def attend(q, K, V, D, see, lam, v_scale, part):
    """One head: q [rows, 128], K, V [keys, 128], D [keys] -> out [rows, 128], how far it may be off, m, l.

    The error of an output is at most: for each key whose 448 P lies so near a rounding border that FP32 may round it the other way, one
    step of its code times |V|; and SUMS of the sum of the absolute terms."""
    S = np.where(see, q @ K.T + D, -np.inf)
    m_all = S.max(1, keepdims=True)
    top = np.where(np.isinf(m_all), 0.0, m_all)
    O, room, size = (np.zeros((len(q), 128)) for _ in range(3))
    l = np.zeros((len(q), 1))
    for blocks in lists_of_blocks(see, part):
        m = np.full_like(top, -np.inf)
        for u in reversed(blocks):
            at = slice(u * 128, min(u * 128 + 128, K.shape[0]))
            m = np.maximum(m, S[:, at].max(1, keepdims=True))
            safe = np.where(np.isinf(m), top, m)
            P = np.exp2(lam * (S[:, at] - safe))
            w = np.where(np.isinf(m), 0.0, np.exp2(lam * (safe - top)))
            hat, step = p_hat(448.0 * P)
            hat, step = np.where(see[:, at], hat, 0.0), np.where(see[:, at], step, 0.0)
            v = np.where(see[:, at].any(0)[:, None], V[at], 0.0)
            l += w * P.sum(1, keepdims=True)
            O += w * (hat @ v)
            room += w * (step @ np.abs(v))
            size += w * (hat @ np.abs(v))
    some = l > 0
    scale = v_scale / (448.0 * np.where(some, l, 1.0))
    return np.where(some, O * scale, 0.0), np.where(some, (room + SUMS * size) * scale, 0.0) + 1e-30, top, l


def lam_of(stats, b, softmax_scale):
    return softmax_scale / np.log(2.0) * float(stats.q_gscale[b]) * float(stats.k_gscale[b])


def evicted(weights, L, keep, sinks, recent):
    """Slots that a head keeps, ascending.  weights: FP32 numpy row."""
    if L <= keep:
        return np.arange(L)
    w = weights.astype(np.float64)
    middle = sorted(range(sinks, L - recent), key=lambda j: (0 if not np.isnan(w[j]) else 1, 0.0 if np.isnan(w[j]) else -w[j], j))
    return np.array(list(range(sinks)) + sorted(middle[:keep - sinks - recent]) + list(range(L - recent, L)))
