"""64-bit references of the calls of kvlinc_bounded.h: rotated rows by complex numbers, attention weights summed over groups, which groups stay."""
import numpy as np
import torch

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


# ---- positions -------------------------------------------------------------------------------------------------------------------
# Tolerance of a rotated number, y = magnitude (x cos a - x' sin a):
#   - the angle: formed in 64 bits, a few 2^-53 of it here and there: 2^-50 |a|; its distance from the nearest quarter of a turn in 32 bits, one rounding of
#     the distance, one of pi / 2, one of their product: 3 * 2^-24 * pi / 4;
#   - sine and cosine: the series' next terms are below 2^-29, its last steps round twice: 2 * 2^-24; the magnitude once, x' sin once, the sum once;
#     together less than 8 * 2^-24 (|x| + |x'|) magnitude;
#   - the result to its type: half a step, eps / 2 |y|, or half of the smallest number's step (2^-24 for binary16).
def rotated(x, positions, freq, interleaved, magnitude):
    """x [..., T, 128] as float64, positions [T]: (y, what it may be off before it is rounded to its type)."""
    x = np.asarray(x, dtype=np.float64)
    c = 2 * len(freq)
    first = np.arange(0, c, 2) if interleaved else np.arange(c // 2)
    second = first + 1 if interleaved else first + c // 2
    angle = np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(freq, dtype=np.float64)
    z = (x[..., first] + 1j * x[..., second]) * (magnitude * np.exp(1j * angle))
    y, off = x.copy(), np.zeros_like(x)
    y[..., first], y[..., second] = z.real, z.imag
    size = abs(magnitude) * (np.abs(x[..., first]) + np.abs(x[..., second])) * (8 * 2.0 ** -24 + 2.0 ** -50 * np.abs(angle))
    off[..., first], off[..., second] = size, size
    return y, off


def rounding(y, dtype):
    return torch.finfo(TYPES[dtype]).eps / 2 * np.abs(y) + (2.0 ** -25 if dtype == "f16" else 0.0)


# ---- accumulated attention weight ---------------------------------------------------------------------------------------------------
# Tolerance of a slot's weight.  A score q K_t = sum_c q_c s_c (code_c - centre) + sum_c q_c (z_c + centre s_c), with A_t = sum_c |q_c| (levels s_c +
# |z_c|) above either sum of its terms' magnitudes, is off by
#   - the products q_c s_c, held in two binary16 numbers, 2^-22 of each, or in four FP8 numbers, 2^-16 of each: with |code - centre| at most half of the
#     levels 2^-17 A_t;
#   - two sums of 128 terms in binary32, a rounding (or truncation, 2^-23) each: 128 * 2^-23 at most, of A_t / 2 for the codes' (the four FP8 terms' sums
#     come to that together), of A_t in 10 roundings for the common part's: less than 2^-17 A_t and 2^-19 A_t;
# so by d = 2^-15 A_t / sqrt(128) at most.  Exponents are binary32 numbers of size E = log2(e) max |score| + 16 (the reference's head room), rounded a few
# times on their way (score, reference, logarithm of a sum, the difference of two): 8 * 2^-24 E ln 2; the exponential and the logarithm themselves
# 2^-22.  An error d of the scores moves a normalised weight by a factor of e^(2 d) at most.  Sums of n weights, none negative: n * 2^-24.
# (Bounds for roundings that all point one way: what random ones of that size come to is compared over all slots, see check_mass.)
def weights(q, keys, positions, group_of, slots, size):
    """Rows q [r, 128] at `positions` over the tokens 0 .. n - 1 with keys [n, 128]; group_of [n]: their slots; size [n, 128]: levels s + |z| of their
    channels (|K| for the window's): (weight of each slot, how far it may be off)."""
    q = np.asarray(q, dtype=np.float64)
    total, off = np.zeros(slots), np.zeros(slots)
    t = np.arange(len(keys))
    for row, p in zip(q, positions):
        if p < 0:
            continue
        s = np.where(t <= p, keys @ row / np.sqrt(128.0), -np.inf)
        w = np.exp(s - s.max())
        w /= w.sum()
        d = 2.0 ** -15 * (size[:p + 1] @ np.abs(row)).max() / np.sqrt(128.0)
        e = 1.4427 * np.abs(s[:p + 1]).max() + 16
        of_slot = np.bincount(group_of, w, minlength=slots)
        total += of_slot
        moved = 2 * (d + 8 * 2.0 ** -24 * e * 0.6932)  # (more than e^7: the weights may be anything)
        off += 1.0 if moved > 7 else of_slot * (np.expm1(moved) + 4 * 2.0 ** -22 + (len(q) + 128) * 2.0 ** -24) + 2.0 ** -60
    return total, off


def slots_of(cache, sizes=None):
    """(slot of every token, number of slots, |channel| sizes) of an oracle cache (oracle.kvcache.build_cache)."""
    nq, n, groups = cache["n_quant"], cache["n"], -(-cache["n_quant"] // 128)
    t = np.arange(n)
    group_of = np.where(t < nq, t // 128, groups)
    levels = 2 ** cache["bits"] - 1
    size = np.zeros((n, 128))
    for j in range(groups):
        size[128 * j:min(128 * j + 128, nq)] = levels * cache["k_scale"][j].astype(np.float64) + np.abs(cache["k_zero"][j].astype(np.float64))
    size[nq:] = np.abs(cache["k_res"].astype(np.float64))
    return group_of, groups + 1, size


def check_mass(got, before, decay, fresh, off, what):
    """One (sequence, KV head)'s slots 0 .. c: every slot within its bound; returns squares of the differences and of the results."""
    want = decay * before + fresh
    d = np.abs(np.asarray(got, dtype=np.float64) - want)
    tol = off + 2 * 2.0 ** -24 * (np.abs(want) + decay * np.abs(before))
    assert (d <= tol).all(), (what, int((d - tol).argmax()), d.max(), tol[(d - tol).argmax()], want[(d - tol).argmax()])
    return float((d ** 2).sum()), float((want ** 2).sum())


# ---- eviction ------------------------------------------------------------------------------------------------------------------------

def stay(mass, n, keep, limit, first, last):
    """Slots that stay of n groups with this mass."""
    if n <= limit:
        return list(range(n))
    fixed = [j for j in range(n) if j < first or j >= n - last]
    key = lambda j: (-np.inf if np.isnan(mass[j]) else mass[j], -j)
    # what is not a number counts as less than any number, minus infinity among them
    others = sorted((j for j in range(n) if j not in set(fixed)), key=lambda j: (not np.isnan(mass[j]),) + key(j), reverse=True)
    return sorted(fixed + others[:keep - len(fixed)])
