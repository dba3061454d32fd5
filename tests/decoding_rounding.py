"""Cases of verification in which 32 bits give another answer than 64: for the oracle with that mistake planted (on the host) and for the kernels.
Every sum and product of 64 bits in them is exact, so that the order of additions and the rounding of 64 bits decide nothing."""
import numpy as np
import torch

import decoding_oracle

KINDS = {"f32": (torch.float32, 24), "f16": (torch.float16, 11), "bf16": (torch.bfloat16, 8)}


def products(kind, count=12):
    """(u, q, p) with u * q < p whose product, rounded to 32 bits, is p: such a token stands, and one whose p is the next number below is refused."""
    bits = KINDS[kind][1]
    grid = 0.5 + np.arange(1, 2 ** min(bits - 1, 10), 2) * 2.0 ** -bits        # q of that type, in [0.5, 1)
    out = []
    for i, q in enumerate(grid):
        if kind == "f32":
            u = np.float32(0.75 + (i + 1) * 2.0 ** -24)
            p = np.float32(np.float64(u) * q)
        else:
            p = q - (i % 40 + 1) * 2.0 ** -bits                               # another number of that type
            if p <= 0.25:
                continue
            u = np.float32(p / q)
        if u < 1 and np.float64(u) * q < np.float64(p) and np.float32(u) * np.float32(q) == np.float32(p):
            out.append((u, np.float32(q), np.float32(p)))
    return out[:: max(1, len(out) // count)][:count]


def below(x, kind):
    """The next number of that type below x, which lies in (0.25, 1)."""
    return np.float32(x) - np.float32(2.0 ** -(KINDS[kind][1] + (1 if x < 0.5 or (x == 0.5) else 0)))


def product_case(kind, v):
    """Two sequences to a product: the first one's token stands, the second one's does not.  target, draft, drafts, uniforms."""
    found = products(kind)
    s, x = 2 * len(found), v // 2
    target, draft = torch.zeros((s, 2, v)), torch.zeros((s, 1, v))
    u = np.zeros((s, 2), np.float32)
    for i, (a, q, p) in enumerate(found):
        target[2 * i, 0, x], target[2 * i + 1, 0, x] = float(p), float(below(p, kind))
        draft[2 * i:2 * i + 2, 0, x] = float(q)
        u[2 * i:2 * i + 2, 0] = a
    target[:, :, v - 1] = 2.0 ** -6
    t = KINDS[kind][0]
    return target.to(t), draft.to(t), np.full((s, 1), x, np.int32), u


def draw_case(kind, v, with_draft):
    """Rows of one 1 and many numbers so small that 32 bits lose them beside it: marks between them.  With a draft the first token is refused and the
    1 loses as small a number."""
    small = 2.0 ** -24 if kind == "f16" else 2.0 ** -26
    step = int(2.0 ** -24 / small)                          # u moves by 2^-24: so many entries
    most = (v - 2) // step - 1
    each = np.unique(np.linspace(1, min(most, 4000), 40).astype(int))
    k, s = int(with_draft), len(each)
    target = torch.full((s, k + 1, v), small)
    target[:, :, 0] = 1.0
    draft, drafts = None, np.zeros((s, k), np.int32)
    if with_draft:
        target[:, 0, 1] = 0.0
        draft = torch.zeros((s, 1, v))
        draft[:, 0, 0] = small
        draft[:, 0, 1] = 0.5
        drafts[:] = 1
    u = np.full((s, k + 1), 0.5, np.float32)
    u[:, -1] = (1.0 - each * 2.0 ** -24).astype(np.float32)
    t = KINDS[kind][0]
    return target.to(t), None if draft is None else draft.to(t), drafts, u


def verify_in_32_bits(target, draft, drafts, uniforms):
    """decoding_oracle.verify with the mistake: products and sums in 32 bits (no counts, tokens inside the vocabulary)."""
    s, k1, v = target.shape
    tokens, accepted = np.full((s, k1), -1, np.int32), np.zeros(s, np.int32)
    f = np.float32
    for i in range(s):
        a = 0
        while a < k1 - 1:
            x = drafts[i, a]
            q = f(1) if draft is None else f(draft[i, a, x])
            if not f(uniforms[i, a]) * q < f(target[i, a, x]):
                break
            tokens[i, a] = x
            a += 1
        p = decoding_oracle.probabilities(target[i, a]).astype(f)
        w = p if a == k1 - 1 else np.maximum(p - draft[i, a].astype(f), f(0))
        c = np.cumsum(w, dtype=f)
        past = np.flatnonzero((c > f(uniforms[i, -1]) * c[-1]) & (w > 0))
        tokens[i, a] = past[0] if past.size else np.flatnonzero(w)[-1]
        accepted[i] = a
    return tokens, accepted
