"""What is measured of the two choices that a decoding step makes among scored candidates: how many drafted tokens
stand against the target's probabilities, and which rows of a cache stand by the attention weight they gathered.

A model that answers in tokens (a detector that writes its boxes out, say) is decoded so: a cheap draft proposes a few
tokens, the target's probabilities settle how many of them stand, and the cache, which grew by the rows that stand, goes
back to its budget.

`own` picks the side: the operators in plain torch operations, or the calls of paper_2502_00535_amd.binding.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


# ---------------------------------------------------------------- cases

def _verify(name, sequences, drafts, vocabulary, type, draft=True, ragged=False, pad=0):
    """`pad`: elements between the end of a row and the start of the next; `draft`: the draft gave probabilities."""
    c = {"kind": "verify", "sequences": sequences, "drafts": drafts, "vocabulary": vocabulary, "type": type, "draft": draft,
         "ragged": ragged, "pad": pad}
    return c if name is None else {"name": name, **c}


def _cache(name, kind, sequences, heads, slots, budget, group=0, tokens=0, type="bf16", row=128, rows="bf16", page=0, ragged=False,
           first=4, recent=64):
    """`kind`: "step" (a decoding step of `tokens` new rows), "prompt" (a prompt of `slots` rows down to the budget), "keep" (the keep
    vector alone, from sums that are there). `group`: query heads to a cached head; `page`: slots to a page, 0: one block a sequence."""
    c = {"kind": kind, "sequences": sequences, "heads": heads, "slots": slots, "budget": budget, "group": group, "tokens": tokens,
         "type": type, "row": row, "rows": rows, "page": page, "ragged": ragged, "first": first, "recent": recent}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # one user's stream: nothing but the cost of a call
        _verify("verify_1x4x32000_f32", 1, 4, 32000, "f32"),
        # a serving batch, probabilities in 16 bits, a large vocabulary
        _verify("verify_32x5x131072_bf16", 32, 5, 131072, "bf16"),
        # drafts looked up in the text (no probabilities of their own), of different lengths, odd rows
        _verify("verify_64x8x50001_f16_lookup", 64, 8, 50001, "f16", draft=False, ragged=True),
        # the largest batch, an odd vocabulary in padded rows
        _verify("verify_256x3x151111_f32", 256, 3, 151111, "f32", ragged=True, pad=17),
        # one user's decoding step: one row more than the budget, one leaves
        _cache("step_1x8x1024_bf16", "step", 1, 8, 1025, 1024, 4, 1, recent=32),
        # a serving batch's step
        _cache("step_64x8x2048_bf16", "step", 64, 8, 2049, 2048, 4, 1),
        # a step after verification: up to five rows stand, pages of sixteen slots, weights in 32 bits
        _cache("step_32x8x4096_paged", "step", 32, 8, 4101, 4096, 4, 5, "f32", page=16, ragged=True),
        # a prompt's cache down to its budget by the weights of the last sixteen tokens
        _cache("prompt_4x8x16384_to_2048", "prompt", 4, 8, 16384, 2048, 4, 16),
        # prompts of different lengths, odd sizes, rows of 80 values
        _cache("prompt_24x4x5003_to_1501", "prompt", 24, 4, 5003, 1501, 2, 8, "f16", row=80, rows="f16", ragged=True, recent=33),
        # one long text
        _cache("prompt_1x8x100003_to_8192", "prompt", 1, 8, 100003, 8192, 4, 32, recent=256),
        # the keep vector for a caller who moves the rows himself, short and long
        _cache("keep_32x16x1999_to_1000", "keep", 32, 16, 1999, 1000, ragged=True),
        _cache("keep_64x8x32768_to_4096", "keep", 64, 8, 32768, 4096),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["verify", "verify", "step", "step", "prompt", "keep"])
    if kind == "verify":
        v = _log_uniform(rng, 1000, 200000)
        k = rng.randint(0, 8)
        return _verify(None, _log_uniform(rng, 1, max(1, min(256, 150_000_000 // (v * (k + 1))))), k, v, rng.choice(list(TYPES)),
                       rng.random() < 0.7, rng.random() < 0.5, rng.choice([0, 0, 1, 24]))
    type, rows = rng.choice(list(TYPES)), rng.choice(["bf16", "f16", "f32"])
    heads, row, page = rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 96, 128]), rng.choice([0, 0, 16, 64])
    ragged, first = rng.random() < 0.5, rng.choice([0, 1, 4])
    if kind == "step":
        budget, tokens = _log_uniform(rng, 128, 8192), rng.choice([1, 1, 1, 4, 7])
        sequences = _log_uniform(rng, 1, max(1, min(128, 1_000_000 // (budget * heads))))
        return _cache(None, kind, sequences, heads, budget + tokens, budget, rng.choice([1, 2, 4, 8]), tokens, type, row, rows, page,
                      ragged, first, budget // rng.choice([4, 16, 64]))
    slots = _log_uniform(rng, 500, 65536)
    budget = max(64, int(slots * rng.choice([0.05, 0.1, 0.25, 0.5])))
    group, tokens = rng.choice([1, 2, 4]), rng.choice([1, 8, 16, 32])
    most = min(400_000, 50_000_000 // (group * tokens)) if kind == "prompt" else 16_000_000
    sequences = _log_uniform(rng, 1, max(1, min(64, most // (slots * heads))))
    return _cache(None, kind, sequences, heads, slots, budget, group, tokens, type, row, rows, page, ragged, first, budget // 16)


# ---------------------------------------------------------------- a case's state

def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    return gen


def _verify_inputs(case, seed):
    """Target rows of a peaked softmax, draft rows near them, tokens drawn from the draft rows."""
    gen = _generator(seed)
    s, k, v, t = case["sequences"], case["drafts"], case["vocabulary"], TYPES[case["type"]]

    def rows(logits):
        held = torch.empty((s, logits.shape[1], v + case["pad"]), dtype=t, device=DEVICE)
        held.fill_(0.25)
        held[..., :v] = torch.softmax(logits, -1)
        return held[..., :v]
    logits = 3.0 * torch.randn((s, k + 1, v), generator=gen, device=DEVICE)
    target, draft, drafts = rows(logits), None, torch.zeros((s, k), dtype=torch.int32, device=DEVICE)
    near = logits[:, :k] + 0.7 * torch.randn((s, k, v), generator=gen, device=DEVICE)
    del logits
    if k:
        held = rows(near)
        # a token from each row: the largest of value / exponential number
        race = held.float() / torch.empty((s, k, v), device=DEVICE).exponential_(generator=gen)
        drafts = race.argmax(-1).to(torch.int32)
        draft = held if case["draft"] else None
    uniforms = torch.rand((s, k + 1), generator=gen, device=DEVICE)
    counts = torch.randint(0, k + 1, (s,), generator=gen, device=DEVICE, dtype=torch.int32) if case["ragged"] else None
    return {"target": target, "draft": draft, "drafts": drafts, "counts": counts, "uniforms": uniforms}


def _cache_inputs(case, seed):
    """Sums with a few heavy rows, weights that favour the same rows, positions in the order that earlier steps left."""
    gen = _generator(seed)
    s, h, n, budget, kind = case["sequences"], case["heads"], case["slots"], case["budget"], case["kind"]
    out = {"counts": None, "lengths": None, "valid": None, "weights": None, "table": None}
    slot = torch.arange(n, device=DEVICE, dtype=torch.int32)
    liking = 1.5 * torch.randn((s, h, n), generator=gen, device=DEVICE)  # how much a row is looked at, as a logarithm
    if kind == "step":
        t = case["tokens"]
        stands = torch.full((s,), t, dtype=torch.int32, device=DEVICE)
        if case["ragged"]:
            stands = torch.randint(1, t + 1, (s,), generator=gen, device=DEVICE, dtype=torch.int32)
            out["valid"] = stands
        out["counts"] = budget + stands
        out["lengths"] = 4 * budget + stands
        # rows of the budget: some far back, some new, in any order of slots; behind them this step's rows
        old = torch.where(slot[:budget] < budget // 2, 7 * slot[:budget], 4 * budget - budget + slot[:budget])
        mix = torch.rand((s, h, budget), generator=gen, device=DEVICE).argsort(-1)
        new = (4 * budget + slot[:n - budget]).expand(s, h, n - budget)
        out["positions"] = torch.cat([old[mix], new], -1).contiguous()
        sums = (liking + 0.3 * torch.randn((s, h, n), generator=gen, device=DEVICE)).exp() * 0.2
        sums[..., budget:] = 0.0
        out["sums"] = sums
    else:
        if case["ragged"]:
            out["counts"] = torch.randint(n // 2, n + 1, (s,), generator=gen, device=DEVICE, dtype=torch.int32)
        out["positions"] = slot.expand(s, h, n).contiguous()
        out["sums"] = torch.zeros((s, h, n), device=DEVICE) if kind == "prompt" else (liking * 0.8).exp()
    if kind == "keep":
        return out
    g, t = case["group"], case["tokens"]
    held = torch.empty((s, h, g, t, n), dtype=TYPES[case["type"]], device=DEVICE)
    count = torch.full((s,), n, dtype=torch.int32, device=DEVICE) if out["counts"] is None else out["counts"]
    dead = slot >= count[:, None, None, None]
    for i in range(g):
        logits = liking[:, :, None] + torch.randn((s, h, t, n), generator=gen, device=DEVICE)
        held[:, :, i] = torch.softmax(logits.masked_fill(dead, float("-inf")), -1)
    out["weights"] = held
    row, rows, page = case["row"], TYPES[case["rows"]], case["page"]
    if page:
        each = -(-n // page)
        out["table"] = torch.rand((s * each,), generator=gen, device=DEVICE).argsort().to(torch.int32).view(s, each)
        shape = (s * each, h, page, row)
    else:
        shape = (s, h, n, row)
    out["keys"] = torch.randn(shape, generator=gen, device=DEVICE).to(rows)
    out["values"] = torch.randn(shape, generator=gen, device=DEVICE).to(rows)
    return out


def _inputs(case, seed):
    return _verify_inputs(case, seed) if case["kind"] == "verify" else _cache_inputs(case, seed)


def prepare(case, seed):
    st = {"case": case, **_inputs(case, seed)}
    s = case["sequences"]
    if case["kind"] == "verify":
        st["tokens"] = torch.empty((s, case["drafts"] + 1), dtype=torch.int32, device=DEVICE)
        st["accepted"] = torch.empty((s,), dtype=torch.int32, device=DEVICE)
    else:
        st["keep"] = torch.empty((s, case["heads"], case["slots"]), dtype=torch.uint8, device=DEVICE)
        st["kept"] = torch.empty((s,), dtype=torch.int32, device=DEVICE)
        st["places"] = torch.arange(case["slots"], device=DEVICE, dtype=torch.int32)
    if own:
        _prepare_own(st)
    return st


def run(st):
    if own:
        return _run_own(st)
    return _plain_verify(st) if st["case"]["kind"] == "verify" else _plain_cache(st)


def _outputs(st, keep, kept):
    out = {"keep": keep, "kept": kept, "sums": st["sums"]}
    if st["case"]["kind"] != "keep":
        out.update(positions=st["positions"], keys=st["keys"], values=st["values"])
    return out


# ---------------------------------------------------------------- the framework's calls

def _prepare_own(st):
    from paper_2502_00535_amd import binding as nms

    c = st["case"]
    if c["kind"] == "verify":
        size = nms.nms_verify_workspace_bytes(c["vocabulary"], c["sequences"])
    else:
        size = nms.nms_cache_workspace_bytes(c["slots"], c["heads"], c["sequences"], c["budget"])
    st["workspace"] = torch.empty(max(256, size), dtype=torch.uint8, device=DEVICE)
    st["nms"] = nms
    if c["kind"] == "verify":  # a serving loop keeps its buffers and its plan
        st["plan"] = nms.VerifyPlan(st["target"], st["draft"], st["drafts"], st["counts"], c["drafts"], c["vocabulary"], c["sequences"],
                                    st["uniforms"], st["tokens"], st["accepted"], st["workspace"])
    elif c["kind"] == "step":
        st["plan"] = nms.CachePlan(*_evict_arguments(st), **_evict_options(st))


def _evict_arguments(st):
    c = st["case"]
    return (st["sums"], st["positions"], st["counts"], st["lengths"], c["slots"], c["heads"], c["sequences"], c["budget"], c["first"],
            c["recent"], [st["keys"], st["values"]], st["keep"], st["kept"], st["workspace"])


def _evict_options(st):
    return {"weights": st["weights"], "valid_tokens": st["valid"], "page_table": st["table"]}


def _run_own(st):
    c, nms = st["case"], st["nms"]
    if c["kind"] == "verify":
        st["plan"]()
        return {"tokens": st["tokens"], "accepted": st["accepted"]}
    if c["kind"] == "step":
        st["plan"]()
    elif c["kind"] == "prompt":
        _new_prompt(st)
        nms.nms_cache_evict_batched(*_evict_arguments(st), **_evict_options(st))
    else:
        nms.nms_cache_keep_batched(st["sums"], st["positions"], st["counts"], st["lengths"], c["slots"], c["heads"], c["sequences"],
                                   c["budget"], c["first"], c["recent"], st["keep"], st["kept"], None, st["workspace"])
    return _outputs(st, st["keep"], st["kept"])


def _new_prompt(st):
    """What a program does when a prompt comes into the cache: its rows lie in order, and nothing has looked at them yet."""
    st["positions"].copy_(st["places"].expand_as(st["positions"]))
    st["sums"].zero_()


# ---------------------------------------------------------------- the plain form

def _probabilities(x):
    """What is no number, infinite or below nothing counts as nothing."""
    x = x.float()
    return torch.where(torch.isfinite(x) & (x > 0), x, torch.zeros_like(x))


def _plain_verify(st):
    c = st["case"]
    s, k = c["sequences"], c["drafts"]
    target, draft, drafts, u = st["target"], st["draft"], st["drafts"].long(), st["uniforms"].double()
    rows = torch.arange(s, device=DEVICE)
    count = torch.full((s,), k, device=DEVICE) if st["counts"] is None else st["counts"].long()
    if k:
        at = drafts[..., None]
        p = _probabilities(target[:, :k].gather(-1, at)[..., 0]).double()
        q = torch.ones_like(p) if draft is None else _probabilities(draft.gather(-1, at)[..., 0]).double()
        stands = (u[:, :k] * q < p) & (torch.arange(k, device=DEVICE) < count[:, None])
        accepted = stands.long().cumprod(-1).sum(-1)
    else:
        accepted = torch.zeros((s,), dtype=torch.long, device=DEVICE)
    p = _probabilities(target[rows, accepted]).double()
    w = p
    if k:
        refused = (accepted < count)[:, None]
        a = accepted.clamp(max=k - 1)
        if draft is None:
            q = torch.zeros_like(p).scatter_(1, drafts[rows, a][:, None], float("inf"))
        else:
            q = _probabilities(draft[rows, a]).double()
        w = torch.where(refused, (p - q).clamp(min=0.0), p)
        w = torch.where((w > 0).any(-1, keepdim=True), w, p)
    sums = w.cumsum(-1)
    past = (sums > u[:, k:] * sums[:, -1:]) & (w > 0)
    vocabulary = torch.arange(c["vocabulary"], device=DEVICE)
    first = torch.where(past, vocabulary, c["vocabulary"]).amin(-1)
    last = torch.where(w > 0, vocabulary, -1).amax(-1)
    token = torch.where(first < c["vocabulary"], first, last)
    place = torch.arange(k + 1, device=DEVICE)
    tokens = torch.cat([drafts, torch.zeros((s, 1), dtype=torch.long, device=DEVICE)], -1)
    tokens = torch.where(place < accepted[:, None], tokens, torch.where(place == accepted[:, None], token[:, None], -1))
    return {"tokens": tokens.int(), "accepted": accepted.int()}


def _plain_cache(st):
    c = st["case"]
    n, budget = c["slots"], min(c["budget"], c["slots"])
    if c["kind"] == "prompt":
        _new_prompt(st)
    sums, positions, slot = st["sums"], st["positions"], st["places"]
    count = torch.full((c["sequences"],), n, dtype=torch.int32, device=DEVICE) if st["counts"] is None else st["counts"]
    length = count if st["lengths"] is None else st["lengths"]
    kept = count.clamp(max=budget)
    count, length, k = count[:, None, None], length[:, None, None], kept[:, None, None]
    live = slot < count
    if st["weights"] is not None:
        w = st["weights"].double()
        good = torch.isfinite(w)
        if st["valid"] is not None:
            good &= (torch.arange(c["tokens"], device=DEVICE) < st["valid"][:, None])[:, None, None, :, None]
        total = (sums.double() + torch.where(good, w, torch.zeros_like(w)).sum((2, 3))).float()
        sums.copy_(torch.where(live, total, sums))
    # one whole number per row that orders as the choice does: protected, then higher sums, then (a stable sort) lower slots
    bits = (sums + 0.0).view(torch.int32).long()
    bits = torch.where(bits < 0, -(bits + 2 ** 31) - 1, bits)
    bits = torch.where(torch.isnan(sums), -2 ** 33, bits)
    guarded = (positions < c["first"]) | (positions >= length - c["recent"])
    bits = torch.where(guarded, 2 ** 33, bits)
    order = torch.where(live, bits, -2 ** 34).sort(dim=-1, descending=True, stable=True).indices
    keep = torch.zeros_like(live.expand_as(order)).scatter_(-1, order, (slot < k).expand_as(order))
    if c["kind"] == "keep":
        return _outputs(st, keep.to(torch.uint8), kept)
    # the i-th kept row behind the budget goes to the i-th free slot
    free, moves = (slot < k) & ~keep, (slot >= k) & keep
    table = torch.zeros((*order.shape[:2], n + 1), dtype=torch.long, device=DEVICE)
    table.scatter_(-1, torch.where(moves, moves.long().cumsum(-1) - 1, n), slot.long().expand_as(order))
    source = torch.where(free, table.gather(-1, (free.long().cumsum(-1) - 1).clamp(min=0)), slot.long())[..., :budget]
    for name in ("keys", "values"):
        rows = st[name]
        if c["page"]:
            head = torch.arange(c["heads"], device=DEVICE)[:, None]

            def at(i):
                i = i.expand(c["sequences"], c["heads"], budget)
                page = st["table"].long()[:, None].expand(-1, c["heads"], -1).gather(-1, i // c["page"])
                return page, head, i % c["page"]
            rows[at(slot[:budget].long())] = rows[at(source)]
        else:
            rows[:, :, :budget] = rows.gather(2, source[..., None].expand(-1, -1, -1, c["row"]))
    positions[..., :budget] = positions.gather(-1, source)
    sums[..., :budget] = sums.gather(-1, source)
    sums.copy_(torch.where((slot >= k) & live, torch.zeros_like(sums), sums))
    return _outputs(st, keep.to(torch.uint8), kept)


# ---------------------------------------------------------------- from the definition, in 64 bits

def exact(case, seed):
    return _exact_verify(case, seed) if case["kind"] == "verify" else _exact_cache(case, seed)


def _exact_verify(case, seed):
    inputs = _verify_inputs(case, seed)
    s, k = case["sequences"], case["drafts"]
    drafts, u = inputs["drafts"].cpu().numpy(), inputs["uniforms"].cpu().numpy().astype(np.float64)
    counts = np.full(s, k) if inputs["counts"] is None else inputs["counts"].cpu().numpy()
    tokens, accepted = np.full((s, k + 1), -1, np.int32), np.zeros(s, np.int32)

    def row(name, i, j):
        return inputs[name][i, j].cpu().double().numpy()
    for i in range(s):
        a = 0
        while a < counts[i]:
            x = drafts[i, a]
            q = 1.0 if inputs["draft"] is None else float(inputs["draft"][i, a, x])
            if not u[i, a] * q < float(inputs["target"][i, a, x]):
                break
            tokens[i, a] = x
            a += 1
        w = row("target", i, a)
        if a < counts[i]:
            if inputs["draft"] is None:
                left = w.copy()
                left[drafts[i, a]] = 0.0
            else:
                left = np.maximum(w - row("draft", i, a), 0.0)
            w = left if left.any() else w
        places = np.flatnonzero(w)
        c = np.cumsum(w[places])
        tokens[i, a] = places[min(np.searchsorted(c, u[i, k] * c[-1], side="right"), len(places) - 1)]
        accepted[i] = a
    return {"tokens": tokens, "accepted": accepted}


def _exact_cache(case, seed):
    inputs = _cache_inputs(case, seed)
    s, h, n, budget = case["sequences"], case["heads"], case["slots"], case["budget"]
    counts = np.full(s, n) if inputs["counts"] is None else inputs["counts"].cpu().numpy()
    lengths = counts if inputs["lengths"] is None else inputs["lengths"].cpu().numpy()
    positions, sums = inputs["positions"].cpu().numpy(), inputs["sums"].double()
    if inputs["weights"] is not None:
        for i in range(s):
            t = case["tokens"] if inputs["valid"] is None else int(inputs["valid"][i])
            m = int(counts[i])
            sums[i, :, :m] += inputs["weights"][i, :, :, :t, :m].double().sum((1, 2))
    sums = sums.cpu().numpy()
    keep, kept = np.zeros((s, h, n), np.uint8), np.minimum(counts, budget).astype(np.int32)
    new_sums, new_positions, to, fro = sums.copy(), positions.copy(), [], []
    for i in range(s):
        m, k = int(counts[i]), int(kept[i])
        for j in range(h):
            p = positions[i, j, :m]
            guarded = (p < case["first"]) | (p >= lengths[i] - case["recent"])
            held = np.where(guarded, 0.0, sums[i, j, :m]).astype(np.float32)  # the sums as they are held
            keep[i, j, np.lexsort((np.arange(m), -held, ~guarded))[:k]] = 1
            free, moved = np.flatnonzero(keep[i, j, :k] == 0), k + np.flatnonzero(keep[i, j, k:m])
            new_sums[i, j, free], new_positions[i, j, free] = sums[i, j, moved], p[moved]
            new_sums[i, j, k:m] = 0.0
            to.append((i * h + j) * n + free)
            fro.append((i * h + j) * n + moved)
    if case["kind"] == "keep":
        return {"keep": keep, "kept": kept, "sums": sums}
    to, fro = (torch.from_numpy(np.concatenate(x)).to(DEVICE) for x in (to, fro))
    out = {"keep": keep, "kept": kept, "sums": new_sums, "positions": new_positions}
    for name in ("keys", "values"):
        rows = inputs[name]

        def place(i):
            sequence, head, slot = i // (h * n), i // n % h, i % n
            if not case["page"]:
                return sequence, head, slot
            return inputs["table"].long()[sequence, slot // case["page"]], head, slot % case["page"]
        moved = rows.clone()
        moved[place(to)] = rows[place(fro)]
        out[name] = moved
    return out


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    """Each input read once, each output written once. Verification reads one row of the target (and of the draft, where a draft was
    refused: about half of the sequences); eviction reads weights, sums and positions, writes sums and the keep vector, and reads and
    writes the rows that lie behind the budget and stay (of chance, as the weights are: the budget's share of them)."""
    s = case["sequences"]
    if case["kind"] == "verify":
        v, k = case["vocabulary"], case["drafts"]
        rows = 1.5 if case["draft"] and k else 1.0
        return {"bytes": float(s * (rows * v * BYTES[case["type"]] + 20.0 * (k + 1))), "flops": float(s * v * 2.0 * rows)}
    frames, n, budget = s * case["heads"], case["slots"], case["budget"]
    held = 0.75 * n if case["ragged"] and case["kind"] != "step" else float(n)
    moved = frames * (held * 8.0 + n)
    if case["kind"] == "keep":
        return {"bytes": moved, "flops": frames * held}
    queries = case["group"] * case["tokens"]
    if case["kind"] == "step":
        rows = case["tokens"] * 0.5
    else:
        rows = budget * max(0.0, 1.0 - budget / held)
        moved += frames * 8.0 * n  # the new prompt's sums and positions
    if case["kind"] == "step" and case["ragged"]:
        queries *= 0.5 * (case["tokens"] + 1) / case["tokens"]
    moved += frames * (held * (queries * BYTES[case["type"]] + 4.0) + rows * 2 * (2 * case["row"] * BYTES[case["rows"]] + 8.0))
    return {"bytes": moved, "flops": frames * held * (queries + 1.0)}
