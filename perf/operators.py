"""Rotary positions and the quantised KV cache of cached diffusion-LLM serving:
the calls whose speed is measured beside perf/cases.py, and their plain forms.

A case is a dict of plain values:

  op        "rotate"   q and k of a batch rotated at their positions
            "handoff"  packed bf16 rows quantised into the pages of a pool and
                       read back from them, as a request's KV goes from a
                       prefill worker into a quantised cache and on from there
            "attend"   one attention call over a planned batch whose cached
                       rows are quantised and whose fresh rows are written
                       quantised
            "migrate"  the same call, after which the requests' KV is read
                       back from the pages (they move to another worker)
  rotate:   rows, hq, hkv, d (head dim); rot (the dims that rotate),
            interleaved (pairs 2j, 2j + 1 instead of j, j + rot / 2), base,
            scaling ("none", "linear", "ntk", "yarn") by factor beyond
            original positions; positions run up to `far`; dtype; transpose
            (the gradient's direction); fused (q and k are views of one fused
            projection's output)
  others:   fmt ("e4m3": 8 bits, "e2m1": 4 bits; blocks of 32 dims share a
            power of two); heads and batch as in perf/cases.py: `decodes`
            block decodes whose prompts are drawn from LN(ln prompt, sigma),
            clipped to [16, longest], and followed by resp response positions;
            block rows each, at `scattered` positions or in one block;
            prefills, the total lengths of whole prefills; layout, the seed of
            the lengths

Head shapes are those of perf/cases.py.
"""
import math

import numpy as np
import torch

own = False
PAGE = 16
BLOCK = 32  # dims that share a scale
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _rotate(name, rows, hq, hkv, d, *, rot, interleaved=False, base=10000.0, scaling="none", factor=1.0, original=4096, far=4096,
            dtype="bf16", transpose=False, fused=False):
    return dict(name=name, op="rotate", rows=rows, hq=hq, hkv=hkv, d=d, rot=rot, interleaved=interleaved, base=base, scaling=scaling,
                factor=factor, original=original, far=far, dtype=dtype, transpose=transpose, fused=fused)


def _cache(name, op, fmt, hq, hkv, d, *, decodes=0, prompt=500, sigma=0.8, longest=4096, resp=256, block=32, scattered=False,
           prefills="", layout=0):
    return dict(name=name, op=op, fmt=fmt, hq=hq, hkv=hkv, d=d, decodes=decodes, prompt=prompt, sigma=sigma, longest=longest, resp=resp,
                block=block, scattered=scattered, prefills=prefills, layout=layout)


def listed():
    return [
        # one block decode's rows: launch latency
        _rotate("rotate_block", 32, 32, 32, 128, rot=128),
        # a busy decode worker of the GQA model, far positions under a stretched context, views of the fused projection
        _rotate("rotate_decodes_yarn", 1536, 28, 4, 128, rot=128, interleaved=True, scaling="yarn", factor=8.0, original=32768,
                far=262144, fused=True),
        # the rows of a prefill worker's batch
        _rotate("rotate_prefills", 15627, 32, 32, 128, rot=128, fused=True),
        # the gradient's direction, in 32 bits, half of each head
        _rotate("rotate_partial_transposed", 4099, 32, 8, 64, rot=32, base=500000.0, scaling="linear", factor=4.0, far=16384,
                dtype="fp32", transpose=True),
        # disaggregated serving: the KV of a decode batch arrives in bf16, lives in a quantised pool and moves on
        _cache("handoff_e4m3", "handoff", "e4m3", 32, 32, 128, decodes=32, prompt=300, longest=2048),
        _cache("handoff_e2m1", "handoff", "e2m1", 28, 4, 128, decodes=48),
        # one request alone on the GPU, between its prefills
        _cache("one_decode_e4m3", "attend", "e4m3", 32, 32, 128, decodes=1, prompt=795, sigma=0.0),
        # a busy decode worker of each model
        _cache("decodes_mha_e4m3", "attend", "e4m3", 32, 32, 128, decodes=32, prompt=300, longest=2048),
        _cache("decodes_gqa_e4m3", "attend", "e4m3", 28, 4, 128, decodes=48),
        # long cached contexts: bound by HBM
        _cache("long_decodes_e4m3", "attend", "e4m3", 32, 32, 128, decodes=64, prompt=2000, longest=8192, resp=512),
        # decodes beside whole prefills, which are written quantised (odd lengths)
        _cache("mixed_mha_e4m3", "attend", "e4m3", 32, 32, 128, decodes=16, prompt=795, resp=1024, prefills="1819,1201", layout=1),
        # per-token cached decodes of a small-head model over a 4-bit cache, whose requests then move on
        _cache("token_migrate_e2m1", "migrate", "e2m1", 32, 8, 64, decodes=24, prompt=400, scattered=True, layout=3),
    ]


def draw(rng):
    """One more case of the same ranges; costs at most what the largest listed ones do."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        hq, hkv, d = rng.choice([(32, 32, 128), (32, 32, 128), (28, 4, 128), (28, 4, 128), (32, 8, 128), (32, 8, 64), (16, 2, 128), (8, 8, 64)])
        op = rng.choice(["rotate", "handoff", "attend", "attend", "migrate"])
        if op == "rotate":
            scaling = rng.choice(["none", "linear", "ntk", "yarn"])
            c = _rotate("", log_int(1, 15000), hq, hkv, d, rot=rng.choice([d, d, d // 2, d // 4, d * 3 // 4, d - 2 * rng.randint(1, 9)]),
                        interleaved=rng.random() < 0.5, base=rng.choice([10000.0, 500000.0, 1000000.0]), scaling=scaling,
                        factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 32.0]), original=rng.choice([2048, 4096, 8192, 32768]),
                        far=log_int(256, 1 << 20), dtype=rng.choice(["bf16", "bf16", "bf16", "fp16", "fp32"]),
                        transpose=rng.random() < 0.25, fused=rng.random() < 0.5)
        else:
            kind = "decode" if op == "handoff" else rng.choice(["decode", "decode", "mixed", "prefill"])
            block = rng.choice([32, 32, 32, 32, 17, 64, 1]) if kind != "prefill" and op != "handoff" else 32
            count = 0 if kind == "decode" else rng.randint(1, 3)
            c = _cache("", op, rng.choice(["e4m3", "e4m3", "e2m1"]), hq, hkv, d, decodes=0 if kind == "prefill" else log_int(1, 64),
                       prompt=log_int(100, 2000), sigma=rng.choice([0.4, 0.8]), longest=rng.choice([2048, 4096, 8192]),
                       resp=rng.choice([256, 512, 1024]), block=block, scattered=block <= 32 and kind != "prefill" and op != "handoff" and rng.random() < 0.2,
                       prefills=",".join(str(log_int(100, 3500)) for _ in range(count)), layout=rng.randrange(1 << 20))
        del c["name"]
        w = work(c)
        if w["flops"] <= 2.5e11 and w["bytes"] <= 8e8 and (op == "rotate" or _padded(c) <= 10e9):
            return c


# ------------------------------------------------------------------ layout
def _decode_lengths(case):
    rng = np.random.default_rng(case["layout"])
    p = rng.normal(math.log(case["prompt"]), case["sigma"], size=case["decodes"])
    return np.clip(np.rint(np.exp(p)), 16, case["longest"]).astype(np.int64)


def _prefill_lengths(case):
    return [int(x) for x in case["prefills"].split(",") if x]


def _padded(case):
    """Bytes of the plain form's largest intermediates."""
    n = [int(p) + case["resp"] for p in _decode_lengths(case)] or [0]
    m = _prefill_lengths(case) or [0]
    return max(4.0 * len(n) * max(n) * max(case["hkv"] * case["d"], case["hq"] * case["block"]), 4.0 * len(m) * max(m) ** 2 * case["hq"])


def _layout(case, seed):
    """Lengths, row positions and page table of the batch: decodes first, then prefills."""
    rng = np.random.default_rng([case["layout"], seed])
    prompts = _decode_lengths(case)
    kv_len = [int(p) + case["resp"] for p in prompts]
    rows, first = [], []
    for p in prompts:
        if case["scattered"]:
            pos = int(p) + np.sort(rng.choice(case["resp"], size=case["block"], replace=False))
        else:
            pos = int(p) + case["block"] * int(rng.integers(0, case["resp"] // case["block"])) + np.arange(case["block"])
        rows.append(pos)
        first.append(int(pos[0]))
    for n in _prefill_lengths(case):
        kv_len.append(n)
        rows.append(np.arange(n))
        first.append(0)
    pages = [-(-n // PAGE) for n in kv_len]
    pool = sum(pages) + sum(pages) // 8 + 1
    indptr = lambda sizes: np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)  # noqa: E731
    return dict(q_indptr=indptr([len(r) for r in rows]), q_offset=np.asarray(first, np.int32), kv_len=np.asarray(kv_len, np.int32),
                page_indptr=indptr(pages), page_ids=rng.permutation(pool)[:sum(pages)].astype(np.int32), rows=rows, pool=pool)


def _places(lay):
    """(page, slot) of every position of every item, items one after the other, on the GPU."""
    page = np.concatenate([lay["page_ids"][lay["page_indptr"][i] + np.arange(n) // PAGE] for i, n in enumerate(lay["kv_len"])])
    slot = np.concatenate([np.arange(n) % PAGE for n in lay["kv_len"]])
    return torch.from_numpy(page.astype(np.int64)).cuda(), torch.from_numpy(slot.astype(np.int64)).cuda()


def _group(lay, items):
    """Index tables of some items, padded to the longest of them: positions and rows."""
    if not len(items):
        return None
    n, r = lay["kv_len"][items].astype(np.int64), np.diff(lay["q_indptr"])[items].astype(np.int64)
    pages = np.zeros((len(items), int(n.max())), np.int64)
    rows, at = np.zeros((len(items), int(r.max())), np.int64), np.zeros((len(items), int(r.max())), np.int64)
    for k, i in enumerate(items):
        pages[k, :n[k]] = lay["page_ids"][lay["page_indptr"][i] + np.arange(n[k]) // PAGE]
        rows[k] = lay["q_indptr"][i] + np.minimum(np.arange(rows.shape[1]), r[k] - 1)
        at[k] = np.asarray(lay["rows"][i])[np.minimum(np.arange(rows.shape[1]), r[k] - 1)]
    put = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    return dict(pages=put(pages), slots=torch.arange(pages.shape[1], device="cuda") % PAGE, live=put(np.arange(pages.shape[1]) < n[:, None]),
                rows=put(rows), at=put(at), real=put(np.arange(rows.shape[1]) < r[:, None]), item=torch.arange(len(items), device="cuda")[:, None])


# ------------------------------------------------------------------ plain forms
def _quantise(x, fmt):
    """Codes (a byte each, or two to a byte, the even dim in the low half) and scale bytes of x [..., d]."""
    b = x.float().unflatten(-1, (-1, BLOCK))
    amax = b.abs().amax(-1)
    bits = amax.view(torch.int32)
    top, cut = (8, 0x600000) if fmt == "e4m3" else (2, 0x400000)  # the largest code is 1.75 * 2^8 or 1.5 * 2^2
    e = ((bits >> 23) - 127 - top + ((bits & 0x7FFFFF) > cut)).clamp(min=-117)
    y = b * ((127 - e) << 23).view(torch.float32)[..., None]
    if fmt == "e4m3":
        codes = y.to(torch.float8_e4m3fn).view(torch.uint8).flatten(-2)
    else:
        a = y.abs()
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        code = (torch.round(a / step) + torch.where(a < 2, 0.0, torch.where(a < 4, 2.0, 4.0))).to(torch.uint8) | (y.signbit().to(torch.uint8) << 3)
        code = code.flatten(-2)
        codes = code[..., 0::2] | (code[..., 1::2] << 4)
    return codes, (e + 127).to(torch.uint8)


def _values(codes, scales, fmt):
    """What codes and scales stand for, in 32 bits."""
    if fmt == "e4m3":
        c = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
        nibble = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()
        c = table[nibble & 7] * (1 - 2 * (nibble >> 3)).float()
    return (c.unflatten(-1, (-1, BLOCK)) * (scales.int() << 23).view(torch.float32)[..., None]).flatten(-2)


def _frequencies(case):
    """Turning rate of each pair in radians a position, and the factor on cos and sin."""
    rot, s = case["rot"], case["factor"]
    j = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    base = case["base"] * (s ** (rot / (rot - 2)) if case["scaling"] == "ntk" else 1.0)
    f = base ** (-2.0 * j / rot)
    if case["scaling"] == "linear":
        return f / s, 1.0
    if case["scaling"] == "yarn":  # pairs that turn 32 times over the original length keep their rate, those that turn less than once are stretched
        keep = ((case["original"] * f / (2.0 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
        return f * keep + f / s * (1.0 - keep), 0.1 * math.log(s) + 1.0
    return f, 1.0


def _rotated(x, cos, sin, case):
    rot = case["rot"]
    y = x.float()
    lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
    out = y.clone()
    out[..., lo] = y[..., lo] * cos - y[..., hi] * sin
    out[..., hi] = y[..., hi] * cos + y[..., lo] * sin
    return out.to(x.dtype)


def _rotate_plain(state):
    case, t = state["case"], state["t"]
    f, m = _frequencies(case)
    angle = t["positions"].double()[:, None, None] * f
    cos, sin = (torch.cos(angle) * m).float(), (torch.sin(angle) * (-m if case["transpose"] else m)).float()
    return [_rotated(t["q"], cos, sin, case), _rotated(t["k"], cos, sin, case)]


def _attend_group(g, t, fmt, out, lse, hq, hkv, d, scale):
    """Items of like size at once, padded: their rows of out and lse."""
    if g is None:
        return
    def sequence(codes, scales, fresh):
        x = _values(codes[g["pages"], :, g["slots"]], scales[g["pages"], :, g["slots"]], fmt)  # items, positions, heads, d
        x[g["item"], g["at"]] = fresh[g["rows"]].float()  # a padded row repeats the item's last one
        return x.transpose(1, 2)
    items, r = g["rows"].shape
    k = sequence(t["k"], t["k_scale"], t["k_new"])
    q = t["q"][g["rows"]].float().view(items, r, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(items, hkv, -1, d)
    s = (q @ k.transpose(-1, -2).contiguous()) * scale
    del k
    s.masked_fill_(~g["live"][:, None, None, :], -math.inf)
    top = s.amax(-1, keepdim=True)
    s = s.sub_(top).exp_()
    total = s.sum(-1, keepdim=True)
    o = (s @ sequence(t["v"], t["v_scale"], t["v_new"]).contiguous()) / total
    put = lambda x, w: x.view(items, hkv, hq // hkv, r, w).permute(0, 3, 1, 2, 4).reshape(items, r, hq, w)[g["real"]]  # noqa: E731
    out[g["rows"][g["real"]]] = put(o, d).to(out.dtype)
    lse[g["rows"][g["real"]]] = put(top + total.log(), 1)[..., 0]


def _attend_plain(state):
    case, t, fmt = state["case"], state["t"], state["case"]["fmt"]
    for g in state["groups"]:
        _attend_group(g, t, fmt, state["out"], state["lse"], case["hq"], case["hkv"], case["d"], state["scale"])
    page, slot = state["fresh"]
    for x, codes, scales in ((t["k_new"], t["k"], t["k_scale"]), (t["v_new"], t["v"], t["v_scale"])):
        codes[page, :, slot], scales[page, :, slot] = _quantise(x, fmt)


def _store_plain(state):
    t, (page, slot) = state["t"], state["places"]
    for x, codes, scales in ((t["k_packed"], t["k"], t["k_scale"]), (t["v_packed"], t["v"], t["v_scale"])):
        codes[page, :, slot], scales[page, :, slot] = _quantise(x, state["case"]["fmt"])


def _load_plain(state):
    t, (page, slot), fmt = state["t"], state["places"], state["case"]["fmt"]
    return [_values(t["k"][page, :, slot], t["k_scale"][page, :, slot], fmt).bfloat16(), _values(t["v"][page, :, slot], t["v_scale"][page, :, slot], fmt).bfloat16()]


# ------------------------------------------------------------------ inputs
def _normal(gen, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _channels(gen, hkv, d):
    """K's dims differ in size by up to a factor of ten or so."""
    return torch.exp(0.4 * torch.randn((hkv, d), generator=gen, device="cuda"))


def _pool(gen, case, pages, channels):
    d, hkv, fmt = case["d"], case["hkv"], case["fmt"]
    codes = torch.empty((pages, hkv, PAGE, d if fmt == "e4m3" else d // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((pages, hkv, PAGE, d // BLOCK), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 27) // (hkv * PAGE * d))
    for a in range(0, pages, step):
        b = min(pages, a + step)
        codes[a:b], scales[a:b] = _quantise((torch.randn((b - a, hkv, PAGE, d), generator=gen, device="cuda") * channels[:, None]).bfloat16(), fmt)
    return codes, scales


def _tensors(case, lay, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 17)
    if case["op"] == "rotate":
        rows, hq, hkv, d, dtype = case["rows"], case["hq"], case["hkv"], case["d"], DTYPES[case["dtype"]]
        positions = torch.randint(0, case["far"], (rows,), generator=gen, device="cuda", dtype=torch.int32)
        if case["fused"]:  # q, k and v of a row side by side
            x = _normal(gen, rows, hq + 2 * hkv, d, dtype=dtype)
            return dict(q=x[:, :hq], k=x[:, hq:hq + hkv], positions=positions)
        return dict(q=_normal(gen, rows, hq, d, dtype=dtype), k=_normal(gen, rows, hkv, d, dtype=dtype), positions=positions)
    hkv, d = case["hkv"], case["d"]
    ck, cv = _channels(gen, hkv, d), torch.ones((hkv, d), device="cuda")
    t = {}
    t["k"], t["k_scale"] = _pool(gen, case, lay["pool"], ck)
    t["v"], t["v_scale"] = _pool(gen, case, lay["pool"], cv)
    n = int(lay["kv_len"].sum()) if case["op"] == "handoff" else int(lay["q_indptr"][-1])
    names = ("k_packed", "v_packed") if case["op"] == "handoff" else ("k_new", "v_new")
    for name, c in zip(names, (ck, cv)):
        t[name] = (torch.randn((n, hkv, d), generator=gen, device="cuda") * c).bfloat16()
    if case["op"] != "handoff":
        t["q"] = _normal(gen, n, case["hq"], d)
    return t


def prepare(case, seed):
    if case["op"] == "rotate":
        t = _tensors(case, None, seed)
        state = dict(case=case, t=t, out=[torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (t["q"], t["k"])])
        if own:
            from paper_2607_04206_amd import rope
            state["plan"] = rope.plan(rot_dim=case["rot"], interleaved=case["interleaved"], base=case["base"], scaling=case["scaling"],
                                      factor=case["factor"], original_len=case["original"], device=t["q"].device)
        return state
    lay = _layout(case, seed)
    t = _tensors(case, lay, seed)
    state = dict(case=case, lay=lay, t=t)
    if case["op"] in ("handoff", "migrate"):
        state["places"] = _places(lay)
        shape = (int(lay["kv_len"].sum()), case["hkv"], case["d"])
        state["packed"] = [torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    if case["op"] != "handoff":
        rows, count = int(lay["q_indptr"][-1]), case["decodes"]
        state.update(out=torch.empty((rows, case["hq"], case["d"]), dtype=torch.bfloat16, device="cuda"),
                     lse=torch.empty((rows, case["hq"]), dtype=torch.float32, device="cuda"),
                     scale=float(np.float32(1.0 / math.sqrt(case["d"]))), page_ids=torch.from_numpy(lay["page_ids"]).cuda(),
                     groups=[_group(lay, np.arange(count)), _group(lay, np.arange(count, len(lay["kv_len"])))])
        pos = np.concatenate(lay["rows"])
        first = np.repeat(lay["page_indptr"][:-1], np.diff(lay["q_indptr"]))
        state["fresh"] = (torch.from_numpy(lay["page_ids"][first + pos // PAGE].astype(np.int64)).cuda(), torch.from_numpy(pos % PAGE).cuda())
    if own:
        from paper_2607_04206_amd import attn, kv, kvq
        table = dict(kv_len=lay["kv_len"], page_indptr=lay["page_indptr"], page_ids=lay["page_ids"], num_kv_heads=case["hkv"],
                     head_dim=case["d"], num_pool_pages=lay["pool"], device=t["k"].device)
        codes = torch.float8_e4m3fn if case["fmt"] == "e4m3" else torch.uint8
        state["cache"] = kvq.QuantCache(t["k"].view(codes), t["v"].view(codes), t["k_scale"], t["v_scale"])
        if "places" in state:
            state["move"] = kv.plan(**table)
        if case["op"] != "handoff":
            state["plan"] = attn.plan(q_indptr=lay["q_indptr"], q_offset=lay["q_offset"], num_q_heads=case["hq"], sm_scale=state["scale"],
                                      q_pos=np.concatenate(lay["rows"]).astype(np.int32) if case["scattered"] else None, **table)
    return state


# ------------------------------------------------------------------ a pass
def _state(state):
    """The pool: its 8-bit codes and its scales as the numbers they are. (What 4-bit codes stand for comes back from the pages.)"""
    t = state["t"]
    scales = [t[k].view(torch.float8_e8m0fnu) for k in ("k_scale", "v_scale")]
    return scales + ([t[k].view(torch.float8_e4m3fn) for k in ("k", "v")] if state["case"]["fmt"] == "e4m3" else [])


def run(state):
    case, t = state["case"], state["t"]
    if case["op"] == "rotate":
        if not own:
            return _rotate_plain(state)
        from paper_2607_04206_amd import rope
        return list(rope.rotate(state["plan"], t["q"], t["k"], t["positions"], q_out=state["out"][0], k_out=state["out"][1],
                                transpose=case["transpose"]))
    if own:
        from paper_2607_04206_amd import kvq
    out = []
    if case["op"] == "handoff":
        if own:
            kvq.kv_import(state["move"], t["k_packed"], t["v_packed"], state["cache"])
        else:
            _store_plain(state)
    else:
        if own:
            kvq.forward(state["plan"], t["q"], t["k_new"], t["v_new"], state["cache"], state["page_ids"], out=state["out"], lse=state["lse"])
        else:
            _attend_plain(state)
        out = [state["out"], state["lse"]]
    if "places" in state:
        out += list(kvq.kv_export(state["move"], state["cache"], *state["packed"])) if own else _load_plain(state)
    return out + _state(state)


def work(case):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] == "rotate":
        size = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": case["rows"] * (2.0 * size * (hq + hkv) * d + 4.0), "flops": 3.0 * case["rows"] * (hq + hkv) * case["rot"]}
    row = (d if case["fmt"] == "e4m3" else d / 2) + d / BLOCK  # bytes of a quantised row of one head
    lengths = [int(p) + case["resp"] for p in _decode_lengths(case)]
    items = [(case["block"], n) for n in lengths] + [(n, n) for n in _prefill_lengths(case)]
    read_back = 2.0 * hkv * (row + 2 * d) * sum(n for _, n in items)
    if case["op"] == "handoff":  # read packed, write the pages; read the pages, write packed
        return {"bytes": 2.0 * read_back, "flops": 0.0}
    # quantised rows of the context once, the fresh rows and their quantised write, Q, O, the page ids and the LSE
    bytes_ = sum(2.0 * hkv * (row * (n - r) + r * (row + 2 * d)) + 4.0 * d * hq * r + 4.0 * -(-n // PAGE) + 4.0 * hq * r for r, n in items)
    return {"bytes": bytes_ + (read_back if case["op"] == "migrate" else 0.0), "flops": sum(4.0 * r * n * d * hq for r, n in items)}


# ------------------------------------------------------------------ in 64 bits
def _power(e):
    """2^e for whole e, every bit of it (torch.ldexp takes a pow() that may be off by one)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_quantise(x, fmt):
    """x [..., d] rounded to codes under the smallest power of two that takes the block's largest value: codes and powers, as numbers."""
    largest, bits, lowest = (448.0, 3, -6) if fmt == "e4m3" else (6.0, 1, 0)
    b = x.double().unflatten(-1, (-1, BLOCK))
    _, e = torch.frexp(b.abs().amax(-1) / largest)  # amax / largest = f * 2^e with f in [0.5, 1)
    f = _power(e - 1)
    power = torch.where(f * largest >= b.abs().amax(-1), f, 2 * f).clamp(min=2.0 ** -117)
    y = b / power[..., None]
    _, e = torch.frexp(y)
    step = _power((e - 1).clamp(min=lowest) - bits)
    return (torch.round(y / step) * step).flatten(-2), power


def _exact_values(codes, scales, fmt):
    byte = codes.long()
    if fmt == "e2m1":
        byte = torch.stack([byte % 16, byte // 16], -1).flatten(-2)
    bits, bias = (3, 7) if fmt == "e4m3" else (1, 1)
    sign, exponent, fraction = byte >> (7 if fmt == "e4m3" else 3), (byte >> bits) % (16 if fmt == "e4m3" else 4), byte % (1 << bits)
    size = torch.where(exponent > 0, 1.0 + fraction.double() / (1 << bits), 2.0 * fraction.double() / (1 << bits)) * _power(exponent - bias)
    size = torch.where(sign > 0, -size, size)
    return size, _power(scales.long() - 127)


def _product(codes, powers):
    return (codes.unflatten(-1, (-1, BLOCK)) * powers[..., None]).flatten(-2)


def exact(case, seed):
    if case["op"] == "rotate":
        return _exact_rotate(case, seed)
    lay, fmt = _layout(case, seed), case["fmt"]
    t = _tensors(case, lay, seed)
    pools = [_exact_values(t[k], t[k + "_scale"], fmt) for k in ("k", "v")]
    items = range(len(lay["kv_len"]))
    pages = [torch.from_numpy(lay["page_ids"][lay["page_indptr"][i]:lay["page_indptr"][i + 1]].astype(np.int64)).cuda() for i in items]
    starts = np.concatenate([[0], np.cumsum(lay["kv_len"])])
    fresh = [slice(int(starts[i]), int(starts[i + 1])) if case["op"] == "handoff" else slice(int(lay["q_indptr"][i]), int(lay["q_indptr"][i + 1])) for i in items]
    at = [torch.arange(int(n), device="cuda") if case["op"] == "handoff" else torch.from_numpy(np.asarray(p, np.int64)).cuda() for n, p in zip(lay["kv_len"], lay["rows"])]
    bf16 = [t["k_packed"], t["v_packed"]] if case["op"] == "handoff" else [t["k_new"], t["v_new"]]
    seqs = lambda i: [_product(c[pages[i]], p[pages[i]]).transpose(1, 2).flatten(0, 1)[:lay["kv_len"][i]] for c, p in pools]  # noqa: E731
    result = []
    if case["op"] != "handoff":
        result = _exact_attend(case, t, lay, seqs, at, fresh, bf16)
    for i in items:
        for (codes, powers), x in zip(pools, bf16):
            codes[pages[i][at[i] // PAGE], :, at[i] % PAGE], powers[pages[i][at[i] // PAGE], :, at[i] % PAGE] = _exact_quantise(x[fresh[i]], fmt)
    if case["op"] != "attend":
        result += [torch.cat(x) for x in zip(*(seqs(i) for i in items))]
    return result + [p for _, p in pools] + ([c for c, _ in pools] if fmt == "e4m3" else [])


def _exact_attend(case, t, lay, seqs, at, fresh, bf16):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    scale = float(np.float32(1.0 / math.sqrt(d)))
    out = torch.empty((int(lay["q_indptr"][-1]), hq, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((int(lay["q_indptr"][-1]), hq), dtype=torch.float64, device="cuda")
    for i, rows in enumerate(fresh):
        k, v = seqs(i)
        k[at[i]], v[at[i]] = bf16[0][rows].double(), bf16[1][rows].double()
        for h in range(hq):
            g = h // (hq // hkv)
            s = t["q"][rows, h].double() @ k[:, g].t().contiguous() * scale
            lse[rows, h] = torch.logsumexp(s, 1)
            out[rows, h] = torch.exp(s - lse[rows, h, None]) @ v[:, g].contiguous()
    return [out, lse]


def _exact_rotate(case, seed):
    t, rot, s = _tensors(case, None, seed), case["rot"], case["factor"]
    rates, size = [], 1.0
    for j in range(rot // 2):
        f = case["base"] ** (-2.0 * j / rot)
        if case["scaling"] == "linear":
            f = f / s
        elif case["scaling"] == "ntk":
            f = (case["base"] * s ** (rot / (rot - 2.0))) ** (-2.0 * j / rot)
        elif case["scaling"] == "yarn":
            turns = case["original"] * f / (2.0 * math.pi)
            share = min(1.0, max(0.0, (turns - 1.0) / (32.0 - 1.0)))
            f = (1.0 - share) * f / s + share * f
            size = 0.1 * math.log(s) + 1.0
        rates.append(f)
    angle = torch.outer(t["positions"].double(), torch.tensor(rates, dtype=torch.float64, device="cuda"))
    turn = torch.polar(torch.full_like(angle, size), -angle if case["transpose"] else angle)[:, None]
    result = []
    for x in (t["q"], t["k"]):
        y = x.double()
        r = y[..., :rot]
        pairs = r.unflatten(-1, (-1, 2)) if case["interleaved"] else r.unflatten(-1, (2, -1)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2)
        result.append(torch.cat([z, y[..., rot:]], -1))
    return result
