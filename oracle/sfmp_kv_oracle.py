"""CPU oracle of the 8-bit paged key/value cache, its attention, its pages, and the choice of the next token.

Slow numpy in 64 bits, one token, page or sequence at a time, written from the definitions; it shares nothing with the
library.  A pool is a dict of codes (uint8 [layers, pages, heads, 2, 64 * dim]) and scales (float64 [layers, pages, heads, 2]),
tables are dicts of table, lengths and refs."""
import math

import numpy as np

PAGE = 64


def fp8_values():
    """The 256 values of the 8-bit floating-point format (1 sign, 4 exponent, 3 mantissa bits, bias 7, no infinities)."""
    v = np.zeros(256)
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        if e == 15 and m == 7:
            x = math.nan
        v[code] = -x if code & 128 else x
    return v


_FP8 = fp8_values()
_POSITIVE = _FP8[:127]  # ascending


def encode(x, fmt):
    """Codes of x (already divided by the scale): nearest value, ties to the even code, limited to the largest."""
    x = np.asarray(x, dtype=np.float64)
    if fmt == "int8":
        return (np.clip(np.rint(x), -127, 127) + 128).astype(np.uint8)
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def decode(codes, fmt):
    return codes.astype(np.float64) - 128.0 if fmt == "int8" else _FP8[codes]


def scale_for(largest, fmt):
    if not np.isfinite(largest):
        return math.nan
    if largest < 2.0 ** -100:
        return 0.0
    if fmt == "int8":
        return largest / 127.0
    e = math.ceil(math.log2(largest / 448.0))
    while largest > 448.0 * 2.0 ** e:
        e += 1
    while largest <= 448.0 * 2.0 ** (e - 1):
        e -= 1
    return 2.0 ** e


def _turned(block, which, dim):
    """A block of a page as [token, dim]."""
    return block.reshape(PAGE, dim) if which == 0 else block.reshape(dim, PAGE).T


def append(pool, layer, tables, slots, row_start, K, V, fmt):
    """Works on the pool in place.  Codes are computed with the scale rounded to fp32, as it is stored."""
    dim = K.shape[2]
    for b, slot in enumerate(slots):
        rows = range(row_start[b], row_start[b + 1])
        length = int(tables["lengths"][slot])
        before = length - len(rows)
        if not rows:
            continue
        for place in range(max(before, 0) // PAGE, -(-length // PAGE)):
            page = tables["table"][slot, place]
            first = max(max(before, 0) - place * PAGE, 0)
            end = min(length - place * PAGE, PAGE)
            for head in range(K.shape[1]):
                for which, X in ((0, K), (1, V)):
                    x = X[[row_start[b] + place * PAGE + t - before for t in range(first, end)], head].astype(np.float64)
                    block = pool["codes"][layer, page, head, which]
                    held = pool["scales"][layer, page, head, which] if first else 0.0
                    with np.errstate(invalid="ignore"):
                        need = scale_for(np.abs(x).max(), fmt)
                    scale = need if not first or math.isnan(need) else held if math.isnan(held) else max(held, need)
                    scale = float(np.float32(scale))
                    turned = _turned(block, which, dim).copy()
                    if first and scale > held:
                        turned[:first] = encode(decode(turned[:first], fmt) * (held / scale), fmt)
                    if not first:
                        turned[:] = 128 if fmt == "int8" else 0
                    turned[first:end] = encode(x / scale if scale > 0 else np.zeros_like(x), fmt)
                    pool["codes"][layer, page, head, which] = (turned if which == 0 else turned.T).reshape(-1)
                    pool["scales"][layer, page, head, which] = scale


def dense(pool, layer, tables, slot, fmt, dim):
    """(K, V) [tokens, heads, dim] of a sequence."""
    length = int(tables["lengths"][slot])
    heads = pool["codes"].shape[2]
    out = np.zeros((2, length, heads, dim))
    for t in range(length):
        page = tables["table"][slot, t // PAGE]
        for which in (0, 1):
            block = pool["codes"][layer, page, :, which].reshape(heads, *((PAGE, dim) if which == 0 else (dim, PAGE)))
            codes = block[:, t % PAGE] if which == 0 else block[:, :, t % PAGE]
            out[which, t] = decode(codes, fmt) * pool["scales"][layer, page, :, which][:, None]
    return out[0], out[1]


def attention(Q, K, V, scale, window=0, sinks=0):
    """A row at position p sees the tokens j <= p, with a window those with j > p - window or j < sinks.  Rows Q [n, q_heads, dim], the last of a sequence with keys and values [t, heads, dim].  Returns (O, lse, spread, products):
    spread [n, q_heads, dim] is sum w |V| / sum w, products [n, q_heads] the largest scale * sum |Q K| of a seen token
    (what rounding errors are in proportion to)."""
    n, heads, dim = Q.shape
    t, group = K.shape[0], heads // K.shape[1]
    O, spread = np.zeros((n, heads, dim)), np.zeros((n, heads, dim))
    lse, products = np.full((n, heads), -math.inf), np.zeros((n, heads))
    for i in range(n):
        p = t - n + i
        lo = max(0, p - window + 1) if window else 0
        if p < lo:
            continue
        seen = np.r_[0:min(sinks, lo), lo:p + 1]
        for h in range(heads):
            k, v = K[seen, h // group], V[seen, h // group]
            with np.errstate(invalid="ignore"):
                z = scale * (k @ Q[i, h].astype(np.float64))
            products[i, h] = scale * np.max(np.abs(k) @ np.abs(Q[i, h].astype(np.float64)))
            m = z.max()
            w = np.exp(z - m)
            lse[i, h] = m + math.log(w.sum()) if not np.isnan(m) else math.nan
            O[i, h] = w @ v / w.sum()
            spread[i, h] = w @ np.abs(v) / w.sum()
    return O, lse, spread, products


def pages_of(tokens):
    return -(-tokens // PAGE)


def reserve(pool, tables, slots, counts):
    """Works in place; returns the status."""
    table, lengths, refs = tables["table"], tables["lengths"], tables["refs"]
    if any(not 0 <= s < len(lengths) or c < 0 for s, c in zip(slots, counts)):
        return -1
    if any(pages_of(lengths[s] + c) > table.shape[1] for s, c in zip(slots, counts)):
        return -1
    plan, left = [], refs.copy()
    for s, c in zip(slots, counts):
        copy = False
        if lengths[s] % PAGE and c > 0:
            last = table[s, lengths[s] // PAGE]
            copy = left[last] > 1
            left[last] -= copy
        plan.append((copy, pages_of(lengths[s] + c) - pages_of(lengths[s])))
    free = [p for p in range(len(refs)) if refs[p] <= 0]
    wanted = sum(c + m for c, m in plan)
    if wanted > len(free):
        return wanted - len(free)
    for (copy, more), s, c in zip(plan, slots, counts):
        if copy:
            old, new = table[s, lengths[s] // PAGE], free.pop(0)
            pool["codes"][:, new] = pool["codes"][:, old]
            pool["scales"][:, new] = pool["scales"][:, old]
            refs[old] -= 1
            refs[new] = 1
            table[s, lengths[s] // PAGE] = new
        for k in range(more):
            new = free.pop(0)
            refs[new] = 1
            table[s, pages_of(lengths[s]) + k] = new
        lengths[s] += c
    return 0


def fork(tables, parents, children):
    for p, c in zip(parents, children):
        n = pages_of(tables["lengths"][p])
        tables["table"][c, :n] = tables["table"][p, :n]
        for page in tables["table"][p, :n]:
            tables["refs"][page] += 1
        tables["lengths"][c] = tables["lengths"][p]


def free(tables, slots, keep=None):
    for i, s in enumerate(slots):
        kept = min(max(0 if keep is None else keep[i], 0), tables["lengths"][s])
        for page in tables["table"][s, pages_of(kept):pages_of(tables["lengths"][s])]:
            tables["refs"][page] -= 1
        tables["lengths"][s] = kept


def compact(pool, tables):
    refs = tables["refs"]
    n = int((refs > 0).sum())
    holes = [p for p in range(n) if refs[p] <= 0]
    movers = [p for p in range(n, len(refs)) if refs[p] > 0]
    to = {m: h for m, h in zip(movers, holes)}
    for m, h in to.items():
        pool["codes"][:, h] = pool["codes"][:, m]
        pool["scales"][:, h] = pool["scales"][:, m]
        refs[h], refs[m] = refs[m], 0
    for s, length in enumerate(tables["lengths"]):
        for j in range(pages_of(length)):
            tables["table"][s, j] = to.get(int(tables["table"][s, j]), tables["table"][s, j])
    return n


def sample(logits, temperature, top_k, top_p, min_p, u):
    """One row of logits (values that fp32 holds).  Returns (token, log-probability, margin): margin is how near, in shares of the
    whole weight, a threshold or the random number came to deciding otherwise.  At temperature 0 all tokens of the largest logit weigh
    the same in the log-probability, though the first is chosen."""
    x = np.where(np.isnan(logits), -math.inf, logits.astype(np.float64))
    m = x.max()
    if m == -math.inf:
        return -1, -math.inf, 1.0
    order = np.lexsort((np.arange(x.size), -x))
    with np.errstate(invalid="ignore"):
        y = np.where(x == m, 0.0, np.where(x == -math.inf, -math.inf, (x - m) / temperature if temperature > 0 else -math.inf))
    w = np.exp(y)
    w[w < 2.0 ** -32] = 0.0
    total = w.sum()
    w, yo = w[order], y[order]
    sums = np.cumsum(w)
    margin = 1.0
    kept = x.size
    if temperature <= 0:
        kept = 1
    elif top_k > 0:
        kept = min(kept, top_k)
    if top_p < 1.0:
        aim = top_p * sums[kept - 1]
        nucleus = int(np.searchsorted(sums, aim)) + 1
        margin = min(margin, np.abs(sums - aim).min() / total)
        kept = min(kept, nucleus)
    if min_p > 0.0:
        floor = math.log(min(min_p, 1.0))
        margin = min(margin, np.abs(np.where(np.isfinite(yo), yo, 1e9) - floor).min() if min_p < 1.0 else 1.0)
        kept = min(kept, int((yo >= floor).sum()))
    r = u * sums[kept - 1]
    at = int((sums <= r).sum())
    margin = min(margin, np.abs(sums[:kept] - r).min() / total if u > 0 and kept > 1 else 1.0)
    return int(order[at]), float(yo[at] - math.log(total)), float(margin)


def reorder(tables, slots, parents):
    """Works in place: sequence slots[i] becomes what slots[parents[i]] was (a parent outside of the call: empty)."""
    table, lengths, refs = tables["table"], tables["lengths"], tables["refs"]
    before = {s: (table[s].copy(), int(lengths[s])) for s in slots}
    for s in slots:
        for page in before[s][0][:pages_of(before[s][1])]:
            refs[page] -= 1
    for s, p in zip(slots, parents):
        row, length = before[slots[p]] if 0 <= p < len(slots) else (table[s], 0)
        n = pages_of(length)
        table[s, :n] = row[:n]
        lengths[s] = length
        for page in row[:n]:
            refs[page] += 1


def beam_select(logits, scores, choices, weights=None, ended=None, end_token=0):
    """One request: logits [beams, vocab].  Returns ([(value, row, token)] in order, at most `choices`; the logarithm's argument of every row, and
    the sum of |l - m| w in proportion to it, which rounded exponentials err in proportion to)."""
    found, sums, slopes = [], np.ones(len(logits)), np.zeros(len(logits))
    weights = np.ones(len(logits)) if weights is None else weights
    for b, row in enumerate(logits):
        score = float(scores[b])
        if not score > -math.inf:
            continue
        if ended is not None and ended[b]:
            found.append((-score * float(weights[b]), b, end_token, score))
            continue
        x = np.asarray(row, dtype=np.float64)
        x = np.minimum(np.where(np.isnan(x), -math.inf, x), float(np.finfo(np.float32).max))
        m = x.max()
        if m == -math.inf:
            continue
        w = np.exp(x - m)
        sums[b] = w.sum()
        there = w > 0
        slopes[b] = (w[there] * (m - x[there])).sum() / sums[b]
        for t in np.argsort(-x, kind="stable")[:choices]:
            if x[t] > -math.inf:
                value = score + ((x[t] - m) - math.log(sums[b]))
                found.append((-value * float(weights[b]), b, int(t), value))
    found.sort(key=lambda f: f[:3])
    return [(v, b, t) for _, b, t, v in found[:choices]], sums, slopes
