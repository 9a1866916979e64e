"""Where a step's tokens go, timed: what a program that trains a model with an embedding and a mixture of experts calls around the
products and the update.

  sort     apm_sort_tokens: positions sorted by their id (a row of the embedding, an expert), where each row's begin,
           and where each position went
  lookup   apm_lookup_forward: y[t] = scale sum over j of w[t, j] table[ids[t, j]]; an id outside the table counts nothing
  grads    apm_sort_tokens and apm_lookup_backward: with p = t ids_per_token + j,
               dtable[v] = scale sum over p with ids[p] = v of w[p] dy[t],   dw[p] = scale sum over columns of dy[t] table[ids[p]]
  product  apm_grouped_product: the linear layers of a mixture's experts over tokens sorted by expert, group g at
           offsets[g] .. offsets[g+1] - 1,  y[t] = w_g x[t] + b_g,  or with w_g transposed for the gradient of the layer's input
  dropout  apm_dropout_apply: y = residual + x m, m = 1 / (1 - p) or 0 by a random number for each element that is counted out
           (Philox 4x32 of ten rounds) and never stored; the gradient is the same call

Widths, vocabularies and expert counts are those of the 124 M, 1.3 B, 13 B and mixture-of-experts shapes.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "i32": torch.int32, "i64": torch.int64}
SIZE = {"bf16": 2, "f32": 4, "i32": 4, "i64": 8}
MASK = 0xFFFFFFFF


# ---- the cases --------------------------------------------------------------------------------

def listed():
    return [
        # a few tokens to their experts: what a call costs that moves next to nothing
        {"name": "sort_few_tokens", "kind": "sort", "tokens": 8, "per": 2, "rows": 8, "ids": "i32", "spread": "router", "none": 0.0},
        # the tokens of 16 sequences of 1024 by their row of the vocabulary, a tenth of them padding
        {"name": "sort_vocabulary", "kind": "sort", "tokens": 16384, "per": 1, "rows": 50257, "ids": "i64", "spread": "words", "none": 0.1},
        # the embedding of the 1.3 B shape, 16 sequences of 1024 tokens
        {"name": "lookup_embedding_1p3b", "kind": "lookup", "tokens": 16384, "per": 1, "rows": 50257, "cols": 2048, "table": "bf16", "y": "bf16",
         "ids": "i64", "weights": "none", "spread": "words", "none": 0.0, "scale": math.sqrt(2048.0)},
        # an odd number of tokens get the outputs of their two experts back, weighted by the router, in 32 bits
        {"name": "lookup_back_from_experts", "kind": "lookup", "tokens": 8191, "per": 2, "rows": 16382, "cols": 1024, "table": "bf16", "y": "f32",
         "ids": "i32", "weights": "f32", "spread": "places", "none": 0.03, "scale": 1.0},
        # the gradient of the 1.3 B shape's embedding: words as text has them, some in a tenth of all places and most in none
        {"name": "grads_embedding_1p3b", "kind": "grads", "tokens": 16384, "per": 1, "rows": 50257, "cols": 2048, "table": "bf16", "y": "bf16",
         "ids": "i64", "weights": "none", "spread": "words", "none": 0.0, "scale": math.sqrt(2048.0)},
        # bags of three rows with weights of an odd-width table, both gradients, in 32 bits
        {"name": "grads_odd_bags", "kind": "grads", "tokens": 3001, "per": 3, "rows": 30011, "cols": 1001, "table": "f32", "y": "f32",
         "ids": "i32", "weights": "f32", "spread": "words", "none": 0.05, "scale": 0.7},
        # one token's first expert layers: two of 64 experts
        {"name": "product_one_token", "kind": "product", "tokens": 2, "out": 4096, "in": 1024, "groups": 64, "active": 2, "behind": 0,
         "type": "bf16", "bias": False, "transposed": False},
        # the second layer of 64 experts, all of them with tokens, padding behind them
        {"name": "product_64_experts", "kind": "product", "tokens": 8192, "out": 1024, "in": 4096, "groups": 64, "active": 64, "behind": 300,
         "type": "bf16", "bias": True, "transposed": False},
        # 8 experts of the 1.3 B shape's feed-forward size: the largest product here
        {"name": "product_8_wide_experts", "kind": "product", "tokens": 16384, "out": 8192, "in": 2048, "groups": 8, "active": 8, "behind": 0,
         "type": "bf16", "bias": True, "transposed": False},
        # the gradient of the input of 64 experts' first layer, an eighth of them with tokens, into 32 bits
        {"name": "product_input_gradient", "kind": "product", "tokens": 8192, "out": 1024, "in": 4096, "groups": 64, "active": 8, "behind": 0,
         "type": "f32", "bias": False, "transposed": True},
        # a block's branch of the 1.3 B shape, dropped out on its way into the residual stream
        {"name": "dropout_branch_1p3b", "kind": "dropout", "rows": 16384, "cols": 2048, "x": "bf16", "y": "bf16", "residual": True, "p": 0.1, "first": 0},
        # the gradient of an odd-width model's dropout, rows in the middle of a longer batch
        {"name": "dropout_odd_gradient", "kind": "dropout", "rows": 777, "cols": 1001, "x": "f32", "y": "bf16", "residual": False, "p": 0.25, "first": 777},
    ]


def _log_between(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    n = _log_between(rng, lo, hi)
    return max(lo, n - n % 64) if rng.random() < 0.5 else n


def draw(rng):
    """One more case of the ranges above: one token up to 16384, odd and even widths, every type, tables of experts and of words."""
    kind = rng.choice(["sort", "lookup", "grads", "grads", "product", "product", "product", "dropout"])
    if kind == "dropout":
        cols = _width(rng, 40, 20480)
        rows = _log_between(rng, 1, min(16384, 16384 * 2048 // cols))
        x, y = rng.choice(["bf16", "bf16", "f32"]), rng.choice(["bf16", "f32"])
        return {"kind": kind, "rows": rows, "cols": cols, "x": x, "y": y, "residual": rng.random() < 0.5 and (x, y) != ("f32", "f32"),
                "p": rng.choice([0.1, 0.1, 0.25, 0.5, 0.0123]), "first": rng.choice([0, rng.randint(1, 1 << 40)])}
    if kind == "product":
        groups = rng.choice([0, 8, 8, 64, 64])
        wide, narrow = _width(rng, 64, 8192), _width(rng, 64, 4096 if groups <= 8 else 1024)
        tokens = _log_between(rng, 1, max(1, min(16384, 16384 * 8192 * 2048 // (wide * narrow))))
        out, k = (wide, narrow) if rng.random() < 0.5 else (narrow, wide)
        return {"kind": kind, "tokens": tokens, "out": out, "in": k, "groups": groups, "active": rng.randint(1, max(1, groups)),
                "behind": rng.choice([0, 0, tokens // 7]) if groups else 0, "type": rng.choice(["bf16", "bf16", "f32"]),
                "bias": rng.random() < 0.5, "transposed": rng.random() < 0.5}
    per = rng.choice([1, 1, 2, 3, 8])
    tokens = _log_between(rng, 1, 16384 // per)
    spread = rng.choice(["words", "words", "router"] if kind == "sort" else ["words", "words", "places"])
    rows = rng.randint(per, 64) if spread == "router" else tokens * per if spread == "places" else _log_between(rng, 8, 50257)
    case = {"kind": kind, "tokens": tokens, "per": per, "rows": rows, "ids": rng.choice(["i32", "i64"]), "spread": spread, "none": rng.choice([0.0, 0.0, 0.1])}
    if kind == "sort":
        return case
    cols = min(_width(rng, 40, 5120), 50257 * 1024 // max(rows, tokens * per))
    return dict(case, cols=cols, table=rng.choice(["bf16", "bf16", "f32"]), y=rng.choice(["bf16", "bf16", "f32"]),
                weights=rng.choice(["none", "f32", "bf16"]) if per > 1 else "none", scale=rng.choice([1.0, 0.7, 32.0]))


def work(case):
    if case["kind"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (SIZE[case["x"]] + SIZE[case["y"]] * (2 if case["residual"] else 1)), "flops": 0}
    if case["kind"] == "product":
        t, o, k = case["tokens"] - case["behind"], case["out"], case["in"]
        live = min(case["active"], t)
        return {"bytes": t * (2 * k + SIZE[case["type"]] * o) + live * o * (2 * k + (2 if case["bias"] else 0)), "flops": 2 * t * o * k}
    n, rows = case["tokens"] * case["per"], case["rows"]
    if case["kind"] == "sort":
        return {"bytes": n * (SIZE[case["ids"]] + 12) + 8 * (rows + 1), "flops": 0}
    # rows of the table that occur, each read once: every place, or the words that are expected among so many
    here = n * (1 - case["none"])
    if case["spread"] == "places":
        seen = int(here)
    else:
        every = sum(1.0 / (i + 2.7) for i in range(rows))
        seen = int(sum(1.0 - math.exp(-here / (every * (i + 2.7))) for i in range(rows)))
    moved = case["tokens"] * case["cols"] * SIZE[case["y"]] + n * SIZE[case["ids"]]
    weighted = 0 if case["weights"] == "none" else n * SIZE[case["weights"]]
    if case["kind"] == "lookup":
        return {"bytes": moved + weighted + seen * case["cols"] * SIZE[case["table"]], "flops": 0}
    back = rows * case["cols"] * SIZE[case["table"]]
    return {"bytes": moved + back + (2 * weighted + seen * case["cols"] * SIZE[case["table"]] if weighted else 0), "flops": 0}


# ---- inputs -----------------------------------------------------------------------------------

def _ids(case, g):
    """[tokens, per] rows of a table."""
    tokens, per, rows = case["tokens"], case["per"], case["rows"]
    if case["spread"] == "places":     # a router's: every row of the experts' outputs belongs to one token
        at = torch.randperm(rows, device=DEV, generator=g).view(tokens, per)
    elif case["spread"] == "router":   # the best few of the experts, some of which are liked more
        liking = torch.randn(rows, device=DEV, generator=g)
        at = torch.topk(torch.randn(tokens, rows, device=DEV, generator=g) + liking, per, dim=1).indices
    else:                              # words: the n-th most frequent in about 1 / n of the places, their rows anywhere
        share = torch.cumsum(1.0 / (torch.arange(rows, device=DEV, dtype=torch.float64) + 2.7), 0)
        u = torch.rand(tokens * per, device=DEV, generator=g, dtype=torch.float64) * share[-1]
        at = torch.randperm(rows, device=DEV, generator=g)[torch.searchsorted(share, u).clamp(max=rows - 1)].view(tokens, per)
    if case["none"]:                   # padding, or what found no room at its expert
        at = torch.where(torch.rand(tokens, per, device=DEV, generator=g) < case["none"], -1, at)
    return at.to(TYPES[case["ids"]])


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case)

    def randn(*shape):
        return torch.randn(*shape, device=DEV, generator=g)

    if case["kind"] == "dropout":
        rows, cols = case["rows"], case["cols"]
        s["data"] = randn(rows, cols).to(TYPES[case["x"]])
        s["stream"] = (3 * randn(rows, cols)).to(TYPES[case["y"]]) if case["residual"] else None
        s["seed"], s["layer"] = (seed * 0x9E3779B97F4A7C15 + 11) % (1 << 64), seed % 48
        s["result"] = torch.empty(rows, cols, dtype=TYPES[case["y"]], device=DEV)
        return s
    if case["kind"] == "product":
        t, o, k, n = case["tokens"], case["out"], case["in"], max(1, case["groups"])
        s["data"] = randn(t, k).to(torch.bfloat16)
        s["weights"] = (torch.randn(n, *((k, o) if case["transposed"] else (o, k)), dtype=torch.bfloat16, device=DEV, generator=g) * k ** -0.5)
        s["shift"] = (0.1 * randn(n, o)).to(torch.bfloat16) if case["bias"] else None
        s["result"] = torch.zeros(t, o, dtype=TYPES[case["type"]], device=DEV)   # rows behind the last group stay so
        s["ends"], s["offsets"] = [0, t], None
        if case["groups"]:             # tokens sorted by expert; the active ones take uneven shares
            live = torch.randperm(n, device=DEV, generator=g)[:case["active"]]
            share = torch.zeros(n, device=DEV, dtype=torch.float64)
            share[live] = torch.rand(case["active"], device=DEV, generator=g, dtype=torch.float64) + 0.2
            at = (torch.cumsum(share, 0) / share.sum() * (t - case["behind"])).round().to(torch.int64).clamp(0, t - case["behind"])
            s["offsets"] = torch.cat([at.new_zeros(1), at])
            s["ends"] = s["offsets"].tolist()
        return s
    s["at"] = _ids(case, g)
    n, rows = case["tokens"] * case["per"], case["rows"]
    if case["kind"] != "lookup":
        s["order"], s["place"], s["token"] = (torch.empty(n, dtype=torch.int32, device=DEV) for _ in range(3))
        s["offsets"] = torch.empty(rows + 1, dtype=torch.int64, device=DEV)
    if case["kind"] == "sort":
        return s
    s["rows_of"] = (0.02 * randn(rows, case["cols"])).to(TYPES[case["table"]])
    s["mix"] = torch.softmax(randn(case["tokens"], case["per"]), 1).to(TYPES[case["weights"]]) if case["weights"] != "none" else None
    s["result"] = torch.empty(case["tokens"], case["cols"], dtype=TYPES[case["y"]], device=DEV)
    if case["kind"] == "grads":
        s["dy"] = (1e-3 * randn(case["tokens"], case["cols"])).to(TYPES[case["y"]])
        s["dtable"], s["dmix"] = torch.empty_like(s["rows_of"]), None if s["mix"] is None else torch.empty_like(s["mix"])
    return s


# ---- one pass ---------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _room(s, size):
    """A workspace, which a program keeps from step to step."""
    if s.get("room") is None:
        s["room"] = torch.empty(max(16, size), dtype=torch.uint8, device=DEV)
    return s["room"]


def _run_own(s):
    import paper_2303_02868_amd as apm

    kind = s["kind"]
    if kind == "dropout":
        apm.apm_dropout_apply(apm.make_dropout(s["data"], s["result"], p=s["p"], seed=s["seed"], layer=s["layer"], first_row=s["first"], residual=s["stream"]))
        return s["result"]
    if kind == "product":
        one = s["offsets"] is None
        product = apm.make_grouped_product(s["data"], s["weights"][0] if one else s["weights"], s["result"], offsets=s["offsets"], bias=s["shift"],
                                           transposed=s["transposed"])
        apm.apm_grouped_product(product, _room(s, apm.apm_grouped_product_workspace_bytes(product)))
        return s["result"]
    if kind == "sort":
        order = apm.make_token_order(s["at"], s["rows"], s["order"], offsets=s["offsets"], place=s["place"], token=s["token"])
        apm.apm_sort_tokens(order, _room(s, apm.apm_sort_tokens_workspace_bytes(order)))
        return s["order"], s["offsets"], s["place"], s["token"]
    lookup = apm.make_lookup(s["at"], s["rows_of"], s["result"], scale=s["scale"], weights=s["mix"])
    if kind == "lookup":
        apm.apm_lookup_forward(lookup)
        return s["result"]
    order = apm.make_token_order(s["at"], s["rows"], s["order"], offsets=s["offsets"])
    grads = apm.make_lookup_grads(lookup, s["dy"], order=order, dtable=s["dtable"], dweights=s["dmix"])
    room = _room(s, max(apm.apm_sort_tokens_workspace_bytes(order), apm.apm_lookup_workspace_bytes(lookup)))
    apm.apm_sort_tokens(order, room)
    apm.apm_lookup_backward(lookup, grads, room)
    return s["dtable"], s["dmix"]


def _kept(words, p):
    """Elements whose 16 bits are not under p, out of the generator's four words for each eight."""
    return torch.stack([words & 0xFFFF, words >> 16], dim=-1).flatten(1) >= round(p * 65536)


def _philox(rows, blocks, first, layer, seed):
    """[rows, blocks, 4] words of 32 bits: the counter is (block, row in two words, layer), the key the seed's two words."""
    row = (first + torch.arange(rows, device=DEV))[:, None].expand(rows, blocks)
    c = torch.arange(blocks, device=DEV).expand(rows, blocks), row & MASK, row >> 32, torch.full((rows, blocks), layer, device=DEV)
    k0, k1 = seed & MASK, seed >> 32
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57         # the low 64 bits, whatever their sign
        c = ((b >> 32) & MASK) ^ c[1] ^ k0, b & MASK, ((a >> 32) & MASK) ^ c[3] ^ k1, a & MASK
        k0, k1 = (k0 + 0x9E3779B9) & MASK, (k1 + 0xBB67AE85) & MASK
    return torch.stack(c, dim=-1)


def _run_plain(s):
    kind = s["kind"]
    if kind == "dropout":
        rows, cols, p = s["rows"], s["cols"], s["p"]
        kept = _kept(_philox(rows, -(-cols // 8), s["first"], s["layer"], s["seed"]), p)[:, :cols]
        y = torch.where(kept, s["data"].float() * (65536 / (65536 - round(p * 65536))), 0.0)
        return (y if s["stream"] is None else y + s["stream"].float()).to(s["result"].dtype)
    if kind == "product":
        y, w = torch.zeros_like(s["result"]), s["weights"] if s["transposed"] else s["weights"].transpose(1, 2)
        x = s["data"].float()
        parts = [x[a:b] @ w[i].float() + (0.0 if s["shift"] is None else s["shift"][i].float()) for i, (a, b) in enumerate(zip(s["ends"], s["ends"][1:])) if b > a]
        y[:s["ends"][-1]] = torch.cat(parts).to(y.dtype)
        return y
    rows, per = s["rows"], s["per"]
    flat = s["at"].flatten()
    there = (flat >= 0) & (flat < rows)
    if kind == "sort":
        key = torch.where(there, flat, rows).to(torch.int64)
        key, order = torch.sort(key, stable=True)
        offsets = torch.searchsorted(key, torch.arange(rows + 1, device=DEV))
        places = torch.where(key < rows, torch.arange(key.numel(), device=DEV), -1).to(torch.int32)
        place = torch.empty_like(places)
        place[order] = places
        order = order.to(torch.int32)
        return order, offsets, place, order // per
    row = torch.where(there, flat, 0).to(torch.int64)
    factor = there.float() if s["mix"] is None else torch.where(there, s["mix"].flatten().float(), 0.0)
    if kind == "lookup":
        picked = s["rows_of"][row].float() * factor[:, None]
        return (picked.view(-1, per, s["cols"]).sum(1) * s["scale"]).to(s["result"].dtype)
    dy = s["dy"].float().repeat_interleave(per, 0)
    dtable = torch.zeros(rows, s["cols"], device=DEV).index_add_(0, row, dy * factor[:, None]) * s["scale"]
    dmix = None
    if s["mix"] is not None:
        dmix = (torch.where(there, (dy * s["rows_of"][row].float()).sum(1), 0.0) * s["scale"]).view_as(s["mix"]).to(s["mix"].dtype)
    return dtable.to(s["dtable"].dtype), dmix


# ---- the definition, in 64 bits ---------------------------------------------------------------

def _random_16(case, s):
    """16 random bits for each element, on the host: the generator as its authors describe it, in whole numbers of 64 bits without sign."""
    import numpy as np

    rows, blocks = case["rows"], -(-case["cols"] // 8)
    low, shift = np.uint64(MASK), np.uint64(32)
    row = (np.arange(rows, dtype=np.uint64) + np.uint64(case["first"])).repeat(blocks)
    left0, right0 = np.tile(np.arange(blocks, dtype=np.uint64), rows), row & low
    left1, right1 = row >> shift, np.full(rows * blocks, s["layer"], dtype=np.uint64)
    key = [s["seed"] % 2 ** 32, s["seed"] // 2 ** 32]
    for _ in range(10):
        first, second = left0 * np.uint64(0xD2511F53), left1 * np.uint64(0xCD9E8D57)
        left0, left1 = (second >> shift) ^ right0 ^ np.uint64(key[0]), (first >> shift) ^ right1 ^ np.uint64(key[1])
        right0, right1 = second & low, first & low
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    words = np.stack([left0, right0, left1, right1], axis=1).astype("<u4")
    return words.view("<u2").reshape(rows, blocks * 8)[:, :case["cols"]].astype(np.int32)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "sort":
        return None
    if case["kind"] == "dropout":
        bound = round(case["p"] * 65536)
        bits = torch.from_numpy(_random_16(case, s)).to(DEV)
        y = s["data"].double() / (1.0 - bound / 65536.0)
        y[bits < bound] = 0.0
        return y if s["stream"] is None else s["stream"].double().add_(y)
    if case["kind"] == "product":
        y = torch.zeros(case["tokens"], case["out"], dtype=torch.float64, device=DEV)
        for g in range(len(s["ends"]) - 1):
            a, b = s["ends"][g], s["ends"][g + 1]
            if a < b:
                w = s["weights"][g].double()
                y[a:b] = torch.mm(s["data"][a:b].double(), w if case["transposed"] else w.t().contiguous())
                if case["bias"]:
                    y[a:b] += s["shift"][g].double()
        return y
    tokens, per, cols, rows = case["tokens"], case["per"], case["cols"], case["rows"]
    table = torch.cat([s["rows_of"].double(), torch.zeros(1, cols, dtype=torch.float64, device=DEV)])    # the last row: none
    at = s["at"].long().clone()
    at[(at < 0) | (at >= rows)] = rows
    w = (torch.ones(tokens, per, device=DEV) if s["mix"] is None else s["mix"]).double() * case["scale"]
    if case["kind"] == "lookup":
        y = torch.zeros(tokens, cols, dtype=torch.float64, device=DEV)
        for j in range(per):
            y += w[:, j, None] * table[at[:, j]]
        return y
    dy = s["dy"].double()
    dtable, dw = torch.zeros_like(table), []
    for j in range(per):
        dtable.index_put_((at[:, j],), w[:, j, None] * dy, accumulate=True)
        dw.append(torch.linalg.vecdot(dy, table[at[:, j]]) * case["scale"])
    return dtable[:rows], None if s["mix"] is None else torch.stack(dw, dim=1)
