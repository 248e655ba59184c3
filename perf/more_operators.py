"""The steps around the attention call of cached diffusion-LLM serving: the page
tables that it reads, and the tokens that come of the logits behind it. The
calls whose speed is measured beside perf/operators.py, and their plain forms.

A case is a dict of plain values:

  op        "tokens"   a token and a confidence for every row of logits, from a
                       given uniform number a row
            "unmask"   which masked rows of each block take their token
            "step"     the two, one after the other: what follows the logits
                       of a decode step
            "build"    page list, positions, slots and items of a batch's rows,
                       from the block table of its requests
            "pages"    requests grow into pages of the free list, the batch's
                       tables are built, and the requests shrink back
  tokens, step:  rows, vocab, dtype; pad (logits between the rows: views of
            a padded buffer); style ("greedy", "temperature", "top_k", "top_p",
            "min_p", or "mixed": each request its own); requests of `block`
            rows share their parameters where per_request; confidence
            ("probability", "margin", "entropy"); peak, how far a row's few
            likely tokens stand out of the others at most; forbid (whether one
            token, the mask, is never taken)
  unmask, step:  block rows an item; lengths ("even", or "ragged": from none
            up to twice as many); masked, the share of masked rows; count and
            threshold, which rows are taken
  unmask:   items
  build, pages:  items requests of the table's `requests`; lengths drawn from
            LN(ln length, sigma), clipped to [1, longest]; block rows an item
            at its end, but prefills whole ones; layout, the seed of the lengths
  pages:    growth, the share of requests that grow
"""
import math

import numpy as np
import torch

own = False
PAGE = 16
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
KINDS = ("probability", "margin", "entropy")


def _tokens(name, rows, vocab, style, *, op="tokens", dtype="bf16", pad=0, block=32, per_request=False, confidence="probability", peak=10.0,
            forbid=True, lengths="even", masked=0.7, count=1, threshold=0.9):
    c = dict(name=name, op=op, rows=rows, vocab=vocab, style=style, dtype=dtype, pad=pad, block=block, per_request=per_request,
             confidence=confidence, peak=peak, forbid=forbid)
    return dict(c, lengths=lengths, masked=masked, count=count, threshold=threshold) if op == "step" else c


def _unmask(name, items, block, *, lengths="even", masked=0.7, count=1, threshold=0.9):
    return dict(name=name, op="unmask", items=items, block=block, lengths=lengths, masked=masked, count=count, threshold=threshold)


def _tables(name, op, requests, items, *, length=500, sigma=0.8, longest=4096, block=32, prefills=0, growth=0.1, layout=0):
    return dict(name=name, op=op, requests=requests, items=items, length=length, sigma=sigma, longest=longest, block=block, prefills=prefills,
                growth=growth, layout=layout)


def listed():
    return [
        # one block decode alone on the GPU: the most likely token of each row and how likely it is
        _tokens("block_greedy", 32, 126464, "greedy"),
        # the logits of a busy decode worker: every row's token, by how sure the whole distribution is
        _tokens("decodes_greedy_entropy", 1536, 152064, "greedy", confidence="entropy"),
        # one row of a request with all filters: latency
        _tokens("one_row_filtered", 1, 152064, "mixed", per_request=True, block=1),
        # a decode worker's batch under a nucleus, each request with its own
        _tokens("decodes_top_p", 1024, 126464, "top_p", per_request=True),
        # 32-bit logits of an odd vocabulary in a padded buffer, top-k and the margin of the first two
        _tokens("decodes_top_k_fp32", 257, 50257, "top_k", dtype="fp32", pad=47, block=17, confidence="margin"),
        # plain temperature over flat distributions, where any token may be taken
        _tokens("decodes_temperature", 512, 32000, "temperature", dtype="fp16", peak=2.0),
        # what follows the logits of a decode batch: tokens, then the rows that take them
        _tokens("decode_step", 384, 126464, "mixed", op="step", per_request=True, threshold=0.9),
        # one block, and the blocks of many workers' requests with some long responses decoded without blocks
        _unmask("unmask_block", 1, 32),
        _unmask("unmask_ragged", 2048, 96, lengths="ragged", count=4),
        # the batch of a busy decode worker; long contexts beside whole prefills
        _tables("build_decodes", "build", 64, 48),
        _tables("build_mixed_long", "build", 512, 256, length=2000, longest=16384, prefills=12, layout=1),
        # requests come and go between two iterations of a large worker
        _tables("pages_worker", "pages", 1024, 256, length=1500, longest=8192, growth=0.1, layout=2),
    ]


def draw(rng):
    """One more case of the same ranges; costs at most what the largest listed ones do."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["tokens", "tokens", "tokens", "tokens", "step", "unmask", "build", "pages"])
        count, threshold = rng.choice([0, 1, 1, 2, 4, 8]), rng.choice([0.5, 0.9, 0.9, 1.5])
        lengths, masked = rng.choice(["even", "ragged"]), rng.choice([0.1, 0.5, 0.9, 1.0])
        if op in ("tokens", "step"):
            c = _tokens("", log_int(1, 1536), log_int(500, 160000), rng.choice(["greedy", "temperature", "top_k", "top_p", "min_p", "mixed", "mixed"]),
                        op=op, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), pad=rng.choice([0, 0, 0, rng.randint(1, 200)]),
                        block=rng.choice([1, 17, 32, 32, 64]), per_request=rng.random() < 0.6, confidence=rng.choice(KINDS),
                        peak=rng.uniform(0.0, 15.0), forbid=rng.random() < 0.7, lengths=lengths, masked=masked, count=count, threshold=threshold)
            if c["rows"] * c["vocab"] > 1.6e8:
                continue
        elif op == "unmask":
            c = _unmask("", log_int(1, 4096), log_int(1, 1024), lengths=lengths, masked=masked, count=count, threshold=threshold)
            if c["items"] * c["block"] > 250000:
                continue
        else:
            requests = log_int(1, 2048)
            items = min(requests, log_int(1, 512))
            c = _tables("", op, requests, items, length=log_int(50, 3000), sigma=rng.choice([0.0, 0.4, 0.8]), longest=rng.choice([2048, 8192, 16384]),
                        block=rng.choice([1, 17, 32, 32, 64]), prefills=min(items, rng.choice([0, 0, 1, 4, 12])), growth=rng.choice([0.0, 0.05, 0.3, 1.0]),
                        layout=rng.randrange(1 << 20))
        del c["name"]
        return c


# ------------------------------------------------------------------ inputs
def _generator(seed, salt):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + salt)


def _params(case, rng):
    """Parameters of one request, or of a call."""
    style = rng.choice(["greedy", "temperature", "top_k", "top_p", "min_p", "all", "all"]) if case["style"] == "mixed" else case["style"]
    p = dict(temperature=0.0 if style == "greedy" else float(rng.uniform(0.5, 1.4)), top_k=0, top_p=1.0, min_p=0.0)
    if style in ("top_k", "all"):
        p["top_k"] = int(rng.choice([1, 5, 20, 50, 50, 200, 1000]))
    if style in ("top_p", "all"):
        p["top_p"] = float(rng.choice([0.3, 0.8, 0.9, 0.95, 0.99]))
    if style in ("min_p", "all"):
        p["min_p"] = float(rng.choice([0.01, 0.05, 0.1]))
    return p


NAMES = {"temperature": torch.float32, "top_k": torch.int32, "top_p": torch.float32, "min_p": torch.float32}


def _logits(case, seed):
    """Logits as a language model's last layer gives them: a broad bulk, and a few tokens that stand out by a row's own amount."""
    gen = _generator(seed, 11)
    rows, vocab = case["rows"], case["vocab"]
    buffer = (2.2 * torch.randn((rows, vocab + case["pad"]), generator=gen, device="cuda")).to(DTYPES[case["dtype"]])
    logits = buffer[:, :vocab]
    at = torch.randint(0, vocab, (rows, 24), generator=gen, device="cuda")
    high = 6.0 + case["peak"] * torch.rand((rows, 1), generator=gen, device="cuda") - 3.0 * torch.rand((rows, 24), generator=gen, device="cuda").square()
    # (one column after the other: a token that is drawn twice keeps its last amount)
    again = (at[:, :, None] == at[:, None, :]).triu(1).any(2)
    at = torch.where(again, vocab, at)
    logits.copy_(torch.cat([logits, logits[:, :1]], 1).scatter_(1, at, high.to(logits.dtype))[:, :vocab])
    return logits


def _sampling(case, seed):
    rng = np.random.default_rng([int(seed), 5])
    t = {"logits": _logits(case, seed), "u": torch.rand((case["rows"],), generator=_generator(seed, 13), device="cuda")}
    if case["per_request"]:
        requests = -(-case["rows"] // case["block"])
        each = [_params(case, rng) for _ in range(requests)]
        t["params"] = {k: torch.tensor([p[k] for p in each], dtype=d, device="cuda") for k, d in NAMES.items()}
        t["params_of"] = torch.arange(case["rows"], dtype=torch.int32, device="cuda") // case["block"]
    else:
        t["params"], t["params_of"] = _params(case, rng), None
    t["forbid"] = int(rng.integers(0, case["vocab"])) if case["forbid"] else -1
    return t


def _blocks(case, seed, rows=None):
    """row_indptr of the blocks, ids of their rows (mask_id where masked)."""
    rng = np.random.default_rng([int(seed), 7])
    block = case["block"]
    if rows is None:
        indptr = np.concatenate([[0], np.cumsum(_rows_of_blocks(case))])
    else:
        items = -(-rows // block)
        indptr = np.minimum(np.arange(items + 1) * block, rows)
        if case["lengths"] == "ragged":
            indptr[1:-1] = np.sort(rng.integers(0, rows + 1, items - 1))
    vocab = case.get("vocab", 126464)
    ids = rng.integers(0, vocab, int(indptr[-1]))
    ids[rng.random(len(ids)) < case["masked"]] = vocab  # the mask token: behind the vocabulary's
    put = lambda x: torch.from_numpy(x.astype(np.int32)).cuda()  # noqa: E731
    return {"row_indptr": put(indptr), "ids": put(ids), "mask_id": vocab}


def _lengths(case):
    """Length of every request, the batch's requests and their rows, the requests that grow: the case's, whatever the seed."""
    rng = np.random.default_rng(case["layout"])
    n = np.clip(np.rint(np.exp(rng.normal(math.log(case["length"]), case["sigma"], case["requests"]))), 1, case["longest"]).astype(np.int64)
    request = rng.permutation(case["requests"])[:case["items"]]
    rows, prefill = np.minimum(case["block"], n[request]), np.arange(case["items"]) >= case["items"] - case["prefills"]
    return n, request, np.where(prefill, n[request], rows), rng.random(case["requests"]) < case["growth"]


def _rows_of_blocks(case):
    rng = np.random.default_rng([case["items"], case["block"]])
    return np.full(case["items"], case["block"]) if case["lengths"] == "even" else rng.integers(0, 2 * case["block"] + 1, case["items"])


def _batch(case, seed):
    """Block table, free pages and batch of a worker, the lengths from the case and the places from the seed."""
    places = np.random.default_rng([case["layout"], int(seed)])
    requests = case["requests"]
    n, request, rows, grown = _lengths(case)
    pages = -(-n // PAGE)
    before = np.where(grown, 0, n) if case["op"] == "pages" else n
    held = -(-before // PAGE)
    pool = int(pages.sum()) + int(pages.sum()) // 8 + 1
    order = places.permutation(pool)
    table = np.full((requests, int(pages.max())), -1)
    used = int(held.sum())
    table[np.arange(table.shape[1]) < held[:, None]] = order[:used]
    free = np.full(pool, -1)
    free[:pool - used] = order[used:]
    put = lambda x: torch.from_numpy(np.asarray(x).astype(np.int32)).cuda()  # noqa: E731
    return dict(table=put(table), held=put(held), free=put(free), num_free=put([pool - used]), before=put(before), after=put(n), request=put(request),
                kv_len=put(n[request]), q_indptr=put(np.concatenate([[0], np.cumsum(rows)])), q_offset=put(n[request] - rows), rows=int(rows.sum()),
                pages=int(pages[request].sum()))


def prepare(case, seed):
    if case["op"] in ("build", "pages"):
        return dict(case=case, t=_batch(case, seed))
    if case["op"] == "unmask":
        t = _blocks(case, seed)
        rows, gen = len(t["ids"]), _generator(seed, 17)
        t["tokens"] = torch.randint(0, t["mask_id"], (rows,), generator=gen, device="cuda", dtype=torch.int32)
        # confidences as a decode step gives them: many small ones, some near one, equal ones among them (they came from 8 bits)
        t["confidence"] = torch.rand((rows,), generator=gen, device="cuda").square().bfloat16().float()
        return dict(case=case, t=t)
    t = _sampling(case, seed)
    if case["op"] == "step":
        t.update(_blocks(case, seed, case["rows"]))
    return dict(case=case, t=t)


# ------------------------------------------------------------------ plain forms
def _per_row(t, name, rows):
    """A parameter of each row, a column in 64 bits."""
    x = t["params"][name]
    if not torch.is_tensor(x):
        return torch.full((rows, 1), x, dtype=NAMES[name], device="cuda").double()
    return x[t["params_of"].long()].double()[:, None]


def _tokens_plain(t, kind):
    logits, u = t["logits"], t["u"].double()
    rows, vocab = logits.shape
    temperature, top_k, top_p, min_p = (_per_row(t, k, rows) for k in NAMES)
    x = logits.float()
    if t["forbid"] >= 0:
        x = x.clone()
        x[:, t["forbid"]] = -math.inf
    x, index = torch.sort(x, dim=1, descending=True, stable=True)  # rank order: ties by index
    z = (x.double() - x[:, :1].double()) / torch.where(temperature > 0, temperature, 1.0)
    rank = torch.arange(vocab, device="cuda")[None]
    w = torch.exp(z) * ((rank < top_k) | (top_k == 0))
    before = torch.cumsum(w, 1) - w
    keep = ((before < top_p * w.sum(1, keepdim=True)) & (z >= torch.log(min_p))) | (rank == 0)
    w = w * keep
    mass = w.sum(1, keepdim=True)
    place = (torch.cumsum(w, 1) <= u[:, None] * mass).sum(1, keepdim=True)
    place = torch.minimum(place, (w > 0).sum(1, keepdim=True) - 1) * (temperature > 0)
    if kind == "probability":
        c = w.gather(1, place) / mass
    elif kind == "margin":
        c = (w[:, :1] - w[:, 1:2]) / mass
    else:
        c = torch.where(w > 0, w * z, 0.0).sum(1, keepdim=True) / mass - torch.log(mass)
    return index.gather(1, place)[:, 0].int(), c[:, 0].float()


def _unmask_plain(t, tokens, confidence, count, threshold):
    rows, items = len(t["ids"]), len(t["row_indptr"]) - 1
    item = torch.searchsorted(t["row_indptr"][1:].contiguous(), torch.arange(rows, device="cuda", dtype=torch.int32), right=True)
    candidate = (t["ids"] == t["mask_id"]) & (tokens >= 0) & (tokens != t["mask_id"])
    # rows by item, candidates first, the most confident first, ties by row
    order = torch.sort(torch.where(candidate, confidence, -math.inf), descending=True, stable=True)[1]
    order = order[torch.sort(item[order] * 2 + ~candidate[order], stable=True)[1]]
    rank = torch.empty_like(order)
    rank[order] = torch.arange(rows, device="cuda") - t["row_indptr"].long()[item[order]]
    taken = candidate & ((rank < count) | (confidence >= threshold))
    out = torch.where(taken, tokens, t["ids"])
    left = torch.zeros(items, dtype=torch.int32, device="cuda").index_add_(0, item, (out == t["mask_id"]).int())
    return out, left


def _build_plain(t):
    held = -(-t["kv_len"].long() // PAGE)
    page_indptr = torch.zeros(len(held) + 1, dtype=torch.int32, device="cuda")
    page_indptr[1:] = torch.cumsum(held, 0)
    page = torch.arange(t["pages"], device="cuda")
    item = torch.searchsorted(page_indptr[1:].contiguous(), page.int(), right=True)
    page_ids = t["table"][t["request"].long()[item], page - page_indptr.long()[item]]
    row = torch.arange(t["rows"], device="cuda", dtype=torch.int32)
    item = torch.searchsorted(t["q_indptr"][1:].contiguous(), row, right=True)
    positions = t["q_offset"][item] + row - t["q_indptr"][item]
    slots = t["table"][t["request"].long()[item], positions.long() // PAGE].long() * PAGE + positions % PAGE
    return page_indptr, page_ids, positions, slots, item.int()


def _resize_plain(t, kv_len):
    """The pages of every request follow its length: given back first, then taken, each request's all or none."""
    table, held, free = t["table"], t["held"].long(), t["free"]
    need = -(-kv_len.long() // PAGE)
    column = torch.arange(table.shape[1], device="cuda")[None]
    gives = (column >= need[:, None]) & (column < held[:, None])
    many = t["num_free"].long() + gives.sum()
    # the first request's first page comes out first; entries that do not move go to one behind the last
    place = torch.where(gives, many - torch.cumsum(gives.flatten(), 0).view_as(gives), len(free))
    stack = torch.cat([free, free[:1]]).scatter_(0, place.flatten(), table.flatten())
    wants = (need - held).clamp(min=0)
    fits = torch.cumsum(wants, 0) <= many
    takes = (column < need[:, None]) & (column >= held[:, None]) & fits[:, None]
    place = torch.where(takes, many - torch.cumsum(takes.flatten(), 0).view_as(takes), len(free))
    table.copy_(torch.where(takes, stack[place], torch.where(gives, -1, table)))
    free.copy_(stack[:-1])
    t["held"].copy_(torch.where(fits | (wants == 0), need, held))
    t["num_free"].copy_(many - takes.sum())
    return ((wants > 0) & ~fits).sum(dtype=torch.int32).view(1)


# ------------------------------------------------------------------ a pass
def run(state):
    case, t = state["case"], state["t"]
    if case["op"] in ("tokens", "step"):
        if own:
            from paper_2607_04206_amd import sample
            out = sample.tokens(t["logits"], t["u"], **t["params"], params_of=t["params_of"], confidence=case["confidence"], forbid=t["forbid"])
        else:
            out = _tokens_plain(t, case["confidence"])
        if case["op"] == "tokens":
            return list(out)
        tokens, confidence = out
        blocks = list(out)
    elif case["op"] == "unmask":
        tokens, confidence = t["tokens"], t["confidence"]
        blocks = []
    if case["op"] in ("unmask", "step"):
        if own:
            from paper_2607_04206_amd import sample
            return blocks + list(sample.unmask(tokens, confidence, t["ids"], t["row_indptr"], mask_id=t["mask_id"], count=case["count"],
                                               threshold=case["threshold"]))
        return blocks + list(_unmask_plain(t, tokens, confidence, case["count"], case["threshold"]))
    out = []
    if own:
        from paper_2607_04206_amd import tables
    if case["op"] == "pages":
        out.append(tables.resize(t["table"], t["held"], t["after"], t["free"], t["num_free"]) if own else _resize_plain(t, t["after"]))
    if own:
        b = tables.build(t["table"], t["request"], t["kv_len"], t["q_indptr"], t["q_offset"], rows=t["rows"], pages=t["pages"])
        out += [b.page_indptr, b.page_ids, b.positions, b.slots, b.items]
    else:
        out += _build_plain(t)
    if case["op"] == "pages":
        out.append(tables.resize(t["table"], t["held"], t["before"], t["free"], t["num_free"]) if own else _resize_plain(t, t["before"]))
        out += [t["table"], t["held"], t["free"], t["num_free"]]
    return out


def work(case):
    if case["op"] in ("build", "pages"):
        n, request, rows, grown = _lengths(case)
        b = np.ceil(n[request] / PAGE).sum() * 8 + rows.sum() * 16 + case["items"] * 20
        if case["op"] == "pages":  # a page that moves is read and written on either side, both ways; lengths and pages held are read, the latter written
            b += 2 * (16 * np.ceil(n / PAGE)[grown].sum() + 12 * case["requests"])
        return {"bytes": float(b), "flops": 0.0}
    rows = case["rows"] if "rows" in case else int(_rows_of_blocks(case).sum())
    b, f = 0.0, 0.0
    if case["op"] != "unmask":  # every logit once: a product, an exponential and a sum; tokens and confidences
        size = 4 if case["dtype"] == "fp32" else 2
        b, f = rows * (float(case["vocab"]) * size + 12), 4.0 * rows * case["vocab"]
    if case["op"] != "tokens":
        b += rows * 16 + 8 * -(-rows // case["block"])
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------ in 64 bits
def _exact_row(x, u, kind, temperature, top_k, top_p, min_p):
    """Token and confidence of one row of logits (64 bits, host), by the tokens that can be kept one after the other."""
    top = x.max()
    scaled = (x - top) / (temperature if temperature > 0 else 1.0)
    weight = np.exp(scaled)
    if temperature == 0 and not top_k and top_p >= 1 and min_p <= 0:  # nothing to be ranked but the first two
        token, total = int(np.argmax(x)), math.fsum(weight[weight > 1e-9]) + float(weight[weight <= 1e-9].sum())
        kept = weight
        second = np.partition(weight, -2)[-2] if len(x) > 1 else 0.0
        first = 1.0
    else:
        likely = np.argsort(-x, kind="stable")
        if top_k:
            likely = likely[:top_k]
        mass = np.cumsum(weight[likely])
        number = 1 + int(np.searchsorted(mass, top_p * mass[-1], side="left")) if top_p < 1 else len(likely)
        if min_p > 0:
            number = min(number, int((scaled[likely] >= math.log(min_p)).sum()))
        likely = likely[:max(1, min(number, len(likely)))]
        kept, scaled = weight[likely], scaled[likely]
        total = float(kept.sum())
        at = 0 if temperature == 0 else min(int(np.searchsorted(np.cumsum(kept), u * total, side="right")), int((kept > 0).sum()) - 1)
        token, first, second = int(likely[at]), kept[at], kept[1] if len(kept) > 1 else 0.0
    if kind == "probability":
        return token, first / total
    if kind == "margin":
        return token, (1.0 - second) / total
    return token, float((kept * np.where(kept > 0, scaled, 0.0)).sum()) / total - math.log(total)


def exact(case, seed):
    if case["op"] not in ("tokens", "step"):
        return None
    rows, vocab = case["rows"], case["vocab"]
    if rows * vocab > (3e8 if case["style"] == "greedy" else 1.5e8):
        return None
    t = _sampling(case, seed)
    each = {k: (x[t["params_of"].long()].cpu().double().tolist() if torch.is_tensor(x) else [float(torch.tensor(x, dtype=NAMES[k]))] * rows)
            for k, x in t["params"].items()}
    u = t["u"].double().cpu().tolist()
    tokens, confidence = np.empty(rows, np.int32), np.empty(rows, np.float64)
    for r in range(rows):
        x = t["logits"][r].float().cpu().numpy().astype(np.float64)
        if t["forbid"] >= 0:
            x[t["forbid"]] = -np.inf
        tokens[r], confidence[r] = _exact_row(x, u[r], case["confidence"], each["temperature"][r], int(each["top_k"][r]), each["top_p"][r], each["min_p"][r])
    out = [torch.from_numpy(tokens), torch.from_numpy(confidence)]
    return out if case["op"] == "tokens" else out + [None, None]
