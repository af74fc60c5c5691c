"""The operators of a server that keeps many sequences in one paged cache, as measurable cases.

Three operators that share one pool of pages and one block-table format: rotary
positions with the append of the new keys and values to the pages
(`rope_append`), attention of every sequence's new tokens over its pages
(`paged_attention`), and the pages themselves (`pages_copy`, `pages_fork`,
`pages_extend`, `pages_free`, `pages_compact`).

`run` computes each either through the framework (own) or in plain torch
operations in 32 bits.  Head layouts, page sizes and lengths are those of the
repository's workloads and tests.
"""
import math
import random

import torch

own = False  # whether run() calls the framework's operators

# (d_model, query heads, K/V heads, head size, d_ffn, storage type)
MODELS = {
    "qwen7b": (3584, 28, 4, 128, 18944, "bf16"),
    "qwen15b": (1536, 12, 2, 128, 8960, "bf16"),
    "small64": (768, 12, 2, 64, 2048, "bf16"),
    "tiny": (256, 4, 2, 64, 704, "f32"),
    "tiny128": (312, 3, 1, 128, 520, "f32"),
}
SPARE_PAGES = 4  # pages that no sequence owns


def _dtype(case):
    return torch.bfloat16 if MODELS[case["model"]][5] == "bf16" else torch.float32


def _esz(case):
    return 2 if MODELS[case["model"]][5] == "bf16" else 4


# ----------------------------------------------------------------------------- the cases

def _rope(name, model, seqs, new_lo, new_hi, ctx_lo, ctx_hi, lens_seed, layout="half", rotary=0, theta=1e6,
          scaling="none", factor=1.0, original=0, far=0, page=16, pad=0):
    return {"name": name, "kind": "rope", "model": model, "seqs": seqs, "new_lo": new_lo, "new_hi": new_hi,
            "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "lens_seed": lens_seed, "layout": layout,
            "rotary": rotary or MODELS[model][3], "theta": theta, "scaling": scaling, "factor": factor,
            "original": original, "far": far, "page": page, "pad": pad}


def _attn(name, model, seqs, new_lo, new_hi, ctx_lo, ctx_hi, lens_seed, window=0, lse=False, page=16, pad=0):
    return {"name": name, "kind": "attn", "model": model, "seqs": seqs, "new_lo": new_lo, "new_hi": new_hi,
            "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "lens_seed": lens_seed, "window": window, "lse": lse, "page": page,
            "pad": pad}


def _copy(name, model, layers, pages, page=16):
    return {"name": name, "kind": "copy", "model": model, "layers": layers, "pages": pages, "page": page}


def _branch(name, model, layers, seqs, ctx_lo, ctx_hi, new, lens_seed, page=16):
    return {"name": name, "kind": "branch", "model": model, "layers": layers, "seqs": seqs, "ctx_lo": ctx_lo,
            "ctx_hi": ctx_hi, "new": new, "lens_seed": lens_seed, "page": page}


def _compact(name, model, layers, seqs, ctx_lo, ctx_hi, lens_seed, page=16):
    return {"name": name, "kind": "compact", "model": model, "layers": layers, "seqs": seqs, "ctx_lo": ctx_lo,
            "ctx_hi": ctx_hi, "lens_seed": lens_seed, "page": page}


def listed():
    return [
        # one decoding step of eight short conversations: nothing but latency
        _rope("rope_step15b_8", "qwen15b", 8, 1, 1, 100, 4000, 1),
        # fp32, a few ragged chunks with an idle sequence, interleaved pairs of half the head at far positions
        _rope("rope_f32_ragged", "tiny", 7, 0, 200, 1, 900, 13, layout="interleaved", rotary=32, theta=1e4, far=900000,
              page=8, pad=3),
        # prefill chunks of four long documents past the trained length, scaled by parts
        _rope("rope_chunk7b_16384", "qwen7b", 4, 4096, 4096, 1, 12288, 3, scaling="parts", factor=4.0, original=8192),
        # one user's next token over a short prefix
        _attn("attn_step15b_1", "qwen15b", 1, 1, 1, 3000, 3000, 4),
        # a full server's decoding step, ragged from a question to a long document
        _attn("attn_step7b_64", "qwen7b", 64, 1, 1, 500, 16384, 5),
        # continuous batching: some sequences decode, some bring a chunk of a prompt, one idles; padded rows behind
        _attn("attn_mixed15b_12", "qwen15b", 12, 0, 512, 1, 8192, 6, lse=True, page=32, pad=5),
        # sliding-window chunks at head size 64
        _attn("attn_window64_4", "small64", 4, 500, 2048, 300, 4096, 7, window=1024),
        # the second half of a 16K document in one call
        _attn("attn_prefill7b_8192", "qwen7b", 1, 8192, 8192, 8192, 8192, 8),
        # fp32 storage: a few ragged chunks with their log-sums, small pages
        _attn("attn_f32_6", "tiny", 6, 1, 64, 1, 1500, 9, lse=True, page=8),
        # the window's two layers of a 4K prefix saved before a refresh overwrites them
        _copy("pages_save15b_256", "qwen15b", 2, 256),
        # 32 branches of eight documents: forked, grown by a draft, dropped again
        _branch("pages_branch15b_32", "qwen15b", 28, 32, 500, 4000, 20, 10),
        # half of the sequences have left: the others' pages move together
        _compact("pages_compact15b_24", "qwen15b", 28, 24, 500, 4000, 11),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(max(hi, 1))))))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "step", "step", "draft", "mixed", "mixed", "window", "prefill", "f32", "copy",
                       "branch", "compact"])
    page = rng.choice([16, 16, 16, 32, 64, 8, 1])
    seed = rng.randrange(1 << 20)
    big = rng.choice(["qwen15b", "qwen15b", "qwen7b", "small64"])
    if kind == "rope":
        model = rng.choice([big, "tiny", "tiny128"])
        seqs = _log_int(rng, 1, 64)
        hd = MODELS[model][3]
        scaling = rng.choice(["none", "none", "linear", "base", "parts"])
        c = _rope("", model, seqs, rng.choice([0, 1]), _log_int(rng, 1, 8192 // seqs), 1, _log_int(rng, 2, 8192), seed,
                  layout=rng.choice(["half", "interleaved"]), rotary=rng.choice([hd, hd, hd // 2, hd // 4, 48]),
                  theta=rng.choice([1e4, 1e6]), scaling=scaling, factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.5]),
                  original=4096 if scaling == "parts" else 0, far=rng.choice([0, 0, _log_int(rng, 1000, 1000000)]),
                  page=page, pad=rng.choice([0, 0, 7]))
    elif kind == "step":
        seqs = _log_int(rng, 1, 96)
        c = _attn("", big, seqs, 1, 1, 1, _log_int(rng, 2, 16384), seed, lse=rng.random() < 0.3, page=page)
    elif kind == "draft":
        c = _attn("", big, _log_int(rng, 1, 24), 1, rng.randrange(2, 17), 1, _log_int(rng, 2, 8192), seed,
                  window=rng.choice([0, 0, _log_int(rng, 1, 4096)]), lse=rng.random() < 0.3, page=page)
    elif kind == "mixed":
        c = _attn("", big, _log_int(rng, 2, 16), 0, _log_int(rng, 16, 600), 1, _log_int(rng, 2, 8192), seed,
                  lse=rng.random() < 0.5, page=page, pad=rng.choice([0, 9]))
    elif kind == "window":
        c = _attn("", big, _log_int(rng, 1, 4), 100, _log_int(rng, 101, 2048), 1, _log_int(rng, 2, 4096), seed,
                  window=_log_int(rng, 1, 3000), page=page)
    elif kind == "prefill":
        n = _log_int(rng, 600, 5000)
        c = _attn("", big, 1, n, n, rng.choice([1, 1000, 7000]), _log_int(rng, 7001, 9000), seed, page=page)
    elif kind == "f32":
        c = _attn("", rng.choice(["tiny", "tiny128"]), _log_int(rng, 1, 16), rng.choice([0, 1]), _log_int(rng, 1, 300), 1,
                  _log_int(rng, 2, 3000), seed, window=rng.choice([0, 0, 100]), lse=rng.random() < 0.5, page=page)
    elif kind == "copy":
        c = _copy("", rng.choice(["qwen15b", "qwen7b", "small64", "tiny"]), rng.choice([1, 2, 3, 8]),
                  _log_int(rng, 1, 1024), page=page)
    elif kind == "branch":
        c = _branch("", rng.choice(["qwen15b", "small64", "tiny"]), rng.choice([1, 4, 28]), _log_int(rng, 1, 48), 1,
                    _log_int(rng, 2, 2500), rng.randrange(1, 70), seed, page=page)
    else:
        c = _compact("", rng.choice(["qwen15b", "small64", "tiny"]), rng.choice([1, 4, 28]), _log_int(rng, 1, 48), 1,
                     _log_int(rng, 2, 2000), seed, page=page)
    del c["name"]
    return c


def _lens(case):
    """New tokens and whole lengths of the case's sequences."""
    r = random.Random(case["lens_seed"])
    new, total = [], []
    for s in range(case["seqs"]):
        # (the first brings the most, so that the case has its size whatever is drawn)
        n = case["new_hi"] if s == 0 else _log_int(r, case["new_lo"], case["new_hi"])
        if case["new_lo"] == 0 and s and r.random() < 0.2:
            n = 0
        ctx = case["ctx_hi"] if s == 0 else _log_int(r, case["ctx_lo"], case["ctx_hi"])
        if case["ctx_lo"] <= 1 and s and r.random() < 0.1:
            ctx = 0
        new.append(n)
        total.append(ctx + n)
    return new, total


def _page_lens(case):
    r = random.Random(case["lens_seed"])
    return [case["ctx_hi"] if s == 0 else _log_int(r, case["ctx_lo"], case["ctx_hi"]) for s in range(case["seqs"])]


def _up(a, b):
    return -(-a // b)


def _moved_pages(case):
    """Pages that compaction moves: the live ones past the first `live` of the pool."""
    pages, live = _compact_plan(case)
    return sum(1 for p in live if p >= len(live))


def _compact_plan(case):
    """Pages of each sequence in order of their allocation, and the live ones (of the sequences that stay)."""
    at, pages, live = 0, [], []
    for s, n in enumerate(_page_lens(case)):
        k = _up(n, case["page"])
        pages.append(list(range(at, at + k)))
        if s % 2:  # every second one has left
            live += pages[-1]
        at += k
    return pages, live


def work(case):
    d, nq, nkv, hd, _, _ = MODELS[case["model"]]
    esz = _esz(case)
    if case["kind"] == "rope":
        new, _ = _lens(case)
        rows = sum(new)
        return {"bytes": 2 * rows * (nq + 2 * nkv) * hd * esz, "flops": 3 * rows * (nq + nkv) * case["rotary"]}
    if case["kind"] == "attn":
        new, total = _lens(case)
        w = case["window"]
        keys = pairs = 0
        for n, t in zip(new, total):
            if not n:
                continue
            first = max(0, t - n + 1 - w) if w else 0
            keys += t - first
            seen = lambda p: min(p + 1, w) if w else p + 1  # noqa: E731
            pairs += sum(seen(p) for p in range(t - n, t))
        by = sum(new) * nq * hd * 2 * esz + keys * nkv * hd * 2 * esz + (4 * sum(new) * nq if case["lse"] else 0)
        return {"bytes": by, "flops": 4 * hd * nq * pairs}
    page_bytes = 2 * nkv * case["page"] * hd * esz
    if case["kind"] == "copy":
        return {"bytes": 2 * case["pages"] * case["layers"] * page_bytes + 8 * case["pages"], "flops": 0}
    if case["kind"] == "branch":
        lens = [_page_lens(case)[s % _documents(case)] for s in range(case["seqs"])]
        tails = sum(1 for n in lens if n % case["page"])
        entries = sum(_up(n + case["new"], case["page"]) for n in lens)
        return {"bytes": 2 * tails * case["layers"] * page_bytes + 16 * entries, "flops": 0}
    pages, live = _compact_plan(case)
    return {"bytes": 2 * _moved_pages(case) * case["layers"] * page_bytes + 8 * len(live) + 8 * sum(map(len, pages)),
            "flops": 0}


# ----------------------------------------------------------------------------- inputs

def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + salt) % (1 << 62))
    return g


def _normal(seed, salt, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=_gen(seed, salt), device="cuda", dtype=torch.float32) * scale).to(dtype)


def _normal_pool(seed, salt, shape, dtype):
    pool = torch.empty(shape, device="cuda", dtype=dtype)
    g = _gen(seed, salt)
    for layer in range(shape[0]):
        pool[layer] = torch.randn(shape[1:], generator=g, device="cuda", dtype=torch.float32)
    return pool


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _batch_inputs(case, seed):
    """A ragged batch: row starts, lengths, block tables over shuffled pages, and the pools of two layers."""
    _, nq, nkv, hd, _, _ = MODELS[case["model"]]
    new, total = _lens(case)
    ps = case["page"]
    need = [_up(t, ps) for t in total]
    n_pages = sum(need) + SPARE_PAGES
    width = max(max(need), 1)
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(int(seed)))
    tables = torch.zeros(len(total), width, dtype=torch.int32)
    at = 0
    for s, k in enumerate(need):
        tables[s, :k] = order[at:at + k].to(torch.int32)
        at += k
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    dt = _dtype(case)
    shape = (2, n_pages, nkv, ps, hd)
    return {"rows": starts[-1], "n_rows": starts[-1] + case["pad"], "most_new": max(max(new), 1),
            "row_start": _i32(starts), "length": _i32(total), "tables": tables.cuda(),
            "k_pool": _normal_pool(seed, 1, shape, dt), "v_pool": _normal_pool(seed, 2, shape, dt), "layer": 1}


def _rope_inputs(case, seed):
    _, nq, nkv, hd, _, _ = MODELS[case["model"]]
    x = _batch_inputs(case, seed)
    n = x["n_rows"]
    # the rows of a fused projection: q, k and v are slices of it
    qkv = _normal(seed, 3, (max(n, 1), (nq + 2 * nkv) * hd), _dtype(case))[:n]
    x["q"] = qkv[:, :nq * hd].view(n, nq, hd)
    x["k"] = qkv[:, nq * hd:(nq + nkv) * hd].view(n, nkv, hd)
    x["v"] = qkv[:, (nq + nkv) * hd:].view(n, nkv, hd)
    x["q_out"] = torch.zeros(n, nq, hd, dtype=qkv.dtype, device="cuda")
    # explicit rotary positions where the sequence continues one whose head is no longer cached
    x["positions"] = (torch.arange(n, dtype=torch.int32, device="cuda") + case["far"]) if case["far"] else None
    return x


def _attn_inputs(case, seed):
    _, nq, nkv, hd, _, _ = MODELS[case["model"]]
    x = _batch_inputs(case, seed)
    n = x["n_rows"]
    x["q"] = _normal(seed, 3, (n, nq, hd), _dtype(case), 2.0)
    x["out"] = torch.zeros(n, nq, hd, dtype=_dtype(case), device="cuda")
    x["lse"] = torch.zeros(n, nq, dtype=torch.float32, device="cuda") if case["lse"] else None
    return x


def _copy_inputs(case, seed):
    _, _, nkv, hd, _, _ = MODELS[case["model"]]
    n = case["pages"]
    total = n + n // 2 + SPARE_PAGES
    shape, dt = (case["layers"] + 1, total, nkv, case["page"], hd), _dtype(case)
    order = torch.randperm(total, generator=torch.Generator().manual_seed(int(seed)))
    saved = (case["layers"], n, nkv, case["page"], hd)
    return {"k_pool": _normal_pool(seed, 1, shape, dt), "v_pool": _normal_pool(seed, 2, shape, dt),
            "k_saved": torch.zeros(saved, dtype=dt, device="cuda"), "v_saved": torch.zeros(saved, dtype=dt, device="cuda"),
            "src": order[:n].to(torch.int32).cuda(), "dst": torch.arange(n, dtype=torch.int32, device="cuda")}


def _documents(case):
    return max(1, case["seqs"] // 4)  # four branches of each


def _branch_inputs(case, seed):
    _, _, nkv, hd, _, _ = MODELS[case["model"]]
    ps, docs = case["page"], _documents(case)
    lens = _page_lens(case)[:docs]
    need = [_up(n, ps) for n in lens]
    grown = sum(1 + _up(case["new"], ps) for _ in range(case["seqs"]))
    total = sum(need) + grown + SPARE_PAGES
    width = max(need) + _up(case["new"], ps) + 1
    order = torch.randperm(total, generator=torch.Generator().manual_seed(int(seed)))
    n_seqs = docs + case["seqs"]
    tables = torch.zeros(n_seqs, width, dtype=torch.int32)
    refs = torch.zeros(total, dtype=torch.int32)
    at = 0
    for s, k in enumerate(need):
        tables[s, :k] = order[at:at + k].to(torch.int32)
        refs[order[at:at + k]] = 1
        at += k
    shape, dt = (case["layers"], total, nkv, ps, hd), _dtype(case)
    children = list(range(docs, n_seqs))
    return {"k_pool": _normal_pool(seed, 1, shape, dt), "v_pool": _normal_pool(seed, 2, shape, dt),
            "tables": tables.cuda(), "refs": refs.cuda(), "lengths": _i32(lens + [0] * case["seqs"]),
            "parents": _i32([s % docs for s in range(case["seqs"])]), "children": _i32(children),
            "grow": _i32([0] * docs + [case["new"]] * case["seqs"])}


def _compact_inputs(case, seed):
    _, _, nkv, hd, _, _ = MODELS[case["model"]]
    ps = case["page"]
    lens = _page_lens(case)
    pages, live = _compact_plan(case)
    total = sum(map(len, pages)) + SPARE_PAGES
    width = max(max(map(len, pages)), 1)
    gen = torch.Generator().manual_seed(int(seed))
    tables = torch.zeros(len(lens), width, dtype=torch.int32)
    for s, p in enumerate(pages):  # a sequence's pages in some order of its own
        tables[s, :len(p)] = torch.tensor(p, dtype=torch.int32)[torch.randperm(len(p), generator=gen)]
    refs = torch.zeros(total, dtype=torch.int32)
    refs[torch.tensor(live, dtype=torch.int64)] = torch.randint(1, 4, (len(live),), generator=gen).to(torch.int32)
    shape, dt = (case["layers"], total, nkv, ps, hd), _dtype(case)
    tables, refs = tables.cuda(), refs.cuda()
    return {"k_pool": _normal_pool(seed, 1, shape, dt), "v_pool": _normal_pool(seed, 2, shape, dt), "tables": tables,
            "refs": refs, "lengths": _i32([n if s % 2 else 0 for s, n in enumerate(lens)]),
            # the map after the move; the old one stays valid for work that still reads through it
            "tables_out": torch.zeros_like(tables), "refs_out": torch.zeros_like(refs),
            "remap": torch.zeros_like(refs), "counts": torch.zeros(2, dtype=torch.int32, device="cuda")}


_INPUTS = {"rope": _rope_inputs, "attn": _attn_inputs, "copy": _copy_inputs, "branch": _branch_inputs,
           "compact": _compact_inputs}


def prepare(case, seed):
    x = _INPUTS[case["kind"]](case, seed)
    x["case"] = dict(case)
    if own:  # the handles that a server keeps: the context and the descriptors of its buffers
        _handles(case, x)
    return x


# ----------------------------------------------------------------------------- the framework's calls

def _handles(case, x):
    import paper_2609_30884_amd as crf
    d, nq, nkv, hd, f, dt = MODELS[case["model"]]
    x["crf"] = crf
    dims = crf.make_dims(max(x["k_pool"].shape[0], 1), d, nq, nkv, hd, f, dtype=dt)
    x["ctx"] = crf.Context(dims, 1, 0)
    x["pool"] = crf.page_pool(x["k_pool"], x["v_pool"], case["page"])
    if case["kind"] in ("rope", "attn"):
        x["batch"] = crf.seq_batch(x["row_start"], x["length"], x["tables"], x["n_rows"], x["most_new"])
    if case["kind"] == "rope":
        x["rope"] = crf.rope(case["rotary"], case["theta"], layout=case["layout"], scaling=case["scaling"],
                             factor=case["factor"], original_len=case["original"])
    if case["kind"] == "copy":
        x["saved"] = crf.page_pool(x["k_saved"], x["v_saved"], case["page"])
    if case["kind"] in ("branch", "compact"):
        x["map"] = crf.page_map(x["refs"], x["tables"], x["lengths"], case["page"])
    if case["kind"] == "compact":
        x["map_out"] = crf.page_map(x["refs_out"], x["tables_out"], x["lengths"], case["page"])


def _run_own(x):
    crf, case = x["crf"], x["case"]
    kind = case["kind"]
    if kind == "rope":
        crf.rope_append(x["ctx"], x["rope"], x["batch"], x["q"], x["k"], x["v"], x["pool"], x["layer"], x["q_out"],
                        x["positions"])
    elif kind == "attn":
        crf.paged_attention(x["ctx"], x["batch"], x["q"], x["pool"], x["layer"], x["out"], lse=x["lse"],
                            window=case["window"])
    elif kind == "copy":
        crf.pages_copy(x["ctx"], x["pool"], x["src"], x["dst"], 1, case["layers"], x["saved"], 0)
    elif kind == "branch":
        crf.pages_fork(x["ctx"], x["pool"], x["map"], x["parents"], x["children"])
        crf.pages_extend(x["ctx"], x["map"], x["grow"])
        crf.pages_free(x["ctx"], x["map"], x["children"])
    else:
        crf.pages_compact(x["ctx"], x["pool"], x["map"], x["map_out"], x["remap"], x["counts"])


# ----------------------------------------------------------------------------- the plain forms

def _frequencies(case):
    """Radians per position of each rotated pair, and the factor on cosine and sine."""
    r, s = case["rotary"], case["factor"]
    theta = case["theta"] * s ** (r / (r - 2)) if case["scaling"] == "base" else case["theta"]
    f = torch.arange(0, r, 2, dtype=torch.float64, device="cuda").div(-r).mul(math.log(theta)).exp()
    if case["scaling"] == "linear":
        f = f / s
    if case["scaling"] == "parts":  # pairs of few turns over the trained length are stretched, those of many stay
        g = ((f * case["original"] / (2 * math.pi) - 1.0) / 31.0).clamp(0, 1)
        f = f * ((1 - g) / s + g)
    return f, 0.1 * math.log(s) + 1.0 if case["scaling"] == "parts" else 1.0


def _rows_of(x):
    """Sequence and position of each row."""
    row = torch.arange(x["rows"], device="cuda")
    start = x["row_start"].long()
    seq = (row[:, None] >= start[None, 1:]).sum(1)
    return seq, x["length"].long()[seq] - start[seq + 1] + row


def _rotate(t, cos, sin, r, layout):
    t = t.float()
    a, b = (t[..., 0:r:2], t[..., 1:r:2]) if layout == "interleaved" else (t[..., :r // 2], t[..., r // 2:r])
    x, y = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((x, y), -1).flatten(-2) if layout == "interleaved" else torch.cat((x, y), -1)
    return torch.cat((turned, t[..., r:]), -1)


def _plain_rope(x):
    case, n = x["case"], x["rows"]
    seq, pos = _rows_of(x)
    f, m = _frequencies(case)
    angle = (pos if x["positions"] is None else x["positions"][:n]).double()[:, None] * f
    cos, sin = (angle.cos() * m).float()[:, None], (angle.sin() * m).float()[:, None]
    x["q_out"][:n] = _rotate(x["q"][:n], cos, sin, case["rotary"], case["layout"]).to(x["q"].dtype)
    k = _rotate(x["k"][:n], cos, sin, case["rotary"], case["layout"]).to(x["k"].dtype)
    page, slot = x["tables"][seq, pos // case["page"]].long(), pos % case["page"]
    x["k_pool"][x["layer"]][page, :, slot] = k
    x["v_pool"][x["layer"]][page, :, slot] = x["v"][:n]


def _plain_attn(x):
    """The batch padded to its longest sequence: scores, softmax and products in 32 bits."""
    case, n = x["case"], x["rows"]
    ps, w = case["page"], case["window"]
    seq, pos = _rows_of(x)
    seqs, most = x["tables"].shape[0], x["most_new"]
    nq, hd = x["q"].shape[1:]
    table = x["tables"].long()

    def cached(pool):  # [seqs, kv heads, keys, hd]
        t = pool[x["layer"]][table].float()
        return t.permute(0, 2, 1, 3, 4).reshape(seqs, pool.shape[2], -1, hd)

    k, v = cached(x["k_pool"]), cached(x["v_pool"])
    nkv, keys = k.shape[1], k.shape[2]
    at = torch.arange(n, device="cuda") - x["row_start"].long()[seq]
    q = torch.zeros(seqs, most, nq, hd, device="cuda")
    q[seq, at] = x["q"][:n].float()
    p = torch.zeros(seqs, most, dtype=torch.long, device="cuda")
    p[seq, at] = pos
    g = nq // nkv
    q = q.view(seqs, most, nkv, g, hd).permute(0, 2, 3, 1, 4).reshape(seqs, nkv, g * most, hd)
    s = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(hd)).view(seqs, nkv, g, most, keys)
    j = torch.arange(keys, device="cuda")
    hide = j > p[..., None]
    if w:
        hide |= j <= p[..., None] - w
    s.masked_fill_(hide[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    s.sub_(top).exp_()
    z = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(seqs, nkv, g * most, keys), v).view(seqs, nkv, g, most, hd) / z
    x["out"][:n] = o.permute(0, 3, 1, 2, 4).reshape(seqs, most, nq, hd)[seq, at].to(x["out"].dtype)
    if x["lse"] is not None:
        lse = (top + z.log()).squeeze(-1)
        x["lse"][:n] = lse.permute(0, 3, 1, 2).reshape(seqs, most, nq)[seq, at]


def _plain_copy(x):
    src, dst = x["src"].long(), x["dst"].long()
    x["k_saved"][:, dst] = x["k_pool"][1:, src]
    x["v_saved"][:, dst] = x["v_pool"][1:, src]


def _plain_branch(x):
    ps = x["case"]["page"]
    refs, tables, lengths = x["refs"], x["tables"], x["lengths"]
    parents, children = x["parents"].long(), x["children"].long()
    column = torch.arange(tables.shape[1], device="cuda")
    # fork: the full pages are shared, a page begun is copied to the lowest free one
    n = lengths[parents].long()
    tail = n % ps > 0
    free = (refs == 0).nonzero().squeeze(1)
    fresh = free[(tail.long().cumsum(0) - 1).clamp(min=0)]
    used, full = (n + ps - 1) // ps, n // ps
    rows = tables[parents]
    last = rows.gather(1, (used - 1).clamp(min=0)[:, None]).squeeze(1).long()
    refs.index_add_(0, rows[column < full[:, None]].long(), torch.ones_like(rows[column < full[:, None]]))
    rows = torch.where(tail[:, None] & (column == full[:, None]), fresh[:, None].int(), rows)
    tables[children] = torch.where(column < used[:, None], rows, tables[children])
    lengths[children] = n.int()
    refs[fresh[tail]] = 1
    for pool in (x["k_pool"], x["v_pool"]):
        pool[:, fresh[tail]] = pool[:, last[tail]]
    # extend: the lowest free pages in the order of the sequences
    old = (lengths.long() + ps - 1) // ps
    lengths += x["grow"]
    need = (lengths.long() + ps - 1) // ps - old
    first = need.cumsum(0) - need
    free = (refs == 0).nonzero().squeeze(1)
    nth = first[:, None] + column - old[:, None]
    mine = (column >= old[:, None]) & (column < (old + need)[:, None])
    tables[mine] = free[nth[mine]].int()
    refs[free[nth[mine]]] = 1
    # free
    rows = tables[children]
    gone = rows[column < ((lengths[children].long() + ps - 1) // ps)[:, None]].long()
    refs.index_add_(0, gone, torch.full_like(gone, -1, dtype=torch.int32))
    lengths[children] = 0


def _plain_compact(x):
    ps = x["case"]["page"]
    refs, tables = x["refs"], x["tables"]
    page = torch.arange(refs.numel(), device="cuda")
    live = refs > 0
    n = live.sum()
    moved = (live & (page >= n)).nonzero().squeeze(1)
    hole = (~live & (page < n)).nonzero().squeeze(1)
    remap = torch.where(live, page, -1)
    remap[moved] = hole
    x["remap"].copy_(remap)
    out = torch.where(page < n, refs, 0)
    out[hole] = refs[moved]
    x["refs_out"].copy_(out)
    column = torch.arange(tables.shape[1], device="cuda")
    held = column < ((x["lengths"].long() + ps - 1) // ps)[:, None]
    x["tables_out"].copy_(torch.where(held, remap[tables.long()].int(), x["tables_out"]))
    x["counts"].copy_(torch.stack((n, torch.tensor(moved.numel(), device="cuda"))))
    for pool in (x["k_pool"], x["v_pool"]):
        pool[:, hole] = pool[:, moved]


_PLAIN = {"rope": _plain_rope, "attn": _plain_attn, "copy": _plain_copy, "branch": _plain_branch,
          "compact": _plain_compact}
_OUTPUTS = {"rope": ("q_out", "k_pool", "v_pool"), "attn": ("out", "lse"), "copy": ("k_saved", "v_saved"),
            "branch": ("k_pool", "v_pool", "tables", "refs", "lengths"),
            "compact": ("k_pool", "v_pool", "tables_out", "refs_out", "remap", "counts")}


def run(state):
    if own:
        _run_own(state)
    else:
        _PLAIN[state["case"]["kind"]](state)
    return {name: state[name] for name in _OUTPUTS[state["case"]["kind"]]}


# ----------------------------------------------------------------------------- from the definitions, in 64 bits

def _exact_rope(case, x):
    """Each pair as a complex number times m e^(i angle), row by row of each sequence."""
    new, total = _lens(case)
    r, s = case["rotary"], case["factor"]
    half = r // 2
    freq = []
    for i in range(half):
        base = case["theta"] * (s ** (r / (r - 2)) if case["scaling"] == "base" else 1.0)
        f = base ** (-2.0 * i / r)
        if case["scaling"] == "linear":
            f /= s
        if case["scaling"] == "parts":
            turns = case["original"] * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - 1.0) / (32.0 - 1.0)))
            f = keep * f + (1.0 - keep) * f / s
        freq.append(f)
    freq = torch.tensor(freq, dtype=torch.float64, device="cuda")
    m = 1.0 + 0.1 * math.log(s) if case["scaling"] == "parts" else 1.0
    inter = case["layout"] == "interleaved"
    first = torch.arange(half, device="cuda") * (2 if inter else 1)
    second = first + (1 if inter else half)

    def turn(t, pos):
        t = t.double().clone()
        z = torch.complex(t[..., first], t[..., second]) * torch.polar(torch.full_like(pos[:, None] * freq, m),
                                                                       pos[:, None] * freq)[:, None]
        t[..., first], t[..., second] = z.real, z.imag
        return t

    q_out, kp, vp = x["q_out"].double(), x["k_pool"].double(), x["v_pool"].double()
    row = 0
    for i, (n, t) in enumerate(zip(new, total)):
        if not n:
            continue
        p = torch.arange(t - n, t, device="cuda")
        angle_at = p.double() if not case["far"] else torch.arange(row, row + n, device="cuda").double() + case["far"]
        q_out[row:row + n] = turn(x["q"][row:row + n], angle_at)
        page = x["tables"][i].long()[torch.div(p, case["page"], rounding_mode="floor")]
        kp[x["layer"], page, :, p % case["page"]] = turn(x["k"][row:row + n], angle_at)
        vp[x["layer"], page, :, p % case["page"]] = x["v"][row:row + n].double()
        row += n
    return {"q_out": q_out, "k_pool": kp, "v_pool": vp}


def _exact_attn(case, x):
    """One sequence, K/V head and block of queries at a time."""
    new, total = _lens(case)
    nq, hd = x["q"].shape[1:]
    nkv = x["k_pool"].shape[2]
    g, w = nq // nkv, case["window"]
    out = x["out"].double()
    lse = None if x["lse"] is None else x["lse"].double()
    row = 0
    for i, (n, t) in enumerate(zip(new, total)):
        if not n:
            continue
        key = torch.arange(t, device="cuda")
        page = x["tables"][i].long()[torch.div(key, case["page"], rounding_mode="floor")]
        for h in range(nkv):
            k = x["k_pool"][x["layer"], page, h, key % case["page"]].double()
            v = x["v_pool"][x["layer"], page, h, key % case["page"]].double()
            for b in range(0, n, 1024):
                e = min(n, b + 1024)
                p = torch.arange(t - n + b, t - n + e, device="cuda")[:, None, None]
                q = x["q"][row + b:row + e, h * g:(h + 1) * g].double()
                s = (q.reshape(-1, hd) @ k.t()).view(e - b, g, t) / hd ** 0.5
                seen = (key <= p) & (key > p - w) if w else key <= p
                s = torch.where(seen, s, torch.full_like(s, -math.inf))
                out[row + b:row + e, h * g:(h + 1) * g] = (torch.softmax(s, -1).view(-1, t) @ v).view(e - b, g, hd)
                if lse is not None:
                    lse[row + b:row + e, h * g:(h + 1) * g] = torch.logsumexp(s, -1)
        row += n
    return {"out": out, "lse": lse}


def _exact_copy(case, x):
    k, v = x["k_saved"].double(), x["v_saved"].double()
    for a, b in zip(x["src"].tolist(), x["dst"].tolist()):
        k[:, b] = x["k_pool"][1:, a].double()
        v[:, b] = x["v_pool"][1:, a].double()
    return {"k_saved": k, "v_saved": v}


def _exact_branch(case, x):
    ps = case["page"]
    refs, tables, lengths = x["refs"].tolist(), x["tables"].tolist(), x["lengths"].tolist()
    copies = []
    before = list(refs)
    for a, b in zip(x["parents"].tolist(), x["children"].tolist()):
        n = lengths[a]
        for j in range(n // ps):
            tables[b][j] = tables[a][j]
            refs[tables[a][j]] += 1
        if n % ps:
            p = before.index(0)
            before[p] = refs[p] = 1
            copies.append((tables[a][n // ps], p))
            tables[b][n // ps] = p
        lengths[b] = n
    for s, n in enumerate(x["grow"].tolist()):
        for j in range(_up(lengths[s], ps), _up(lengths[s] + n, ps)):
            tables[s][j] = refs.index(0)
            refs[tables[s][j]] = 1
        lengths[s] += n
    for s in x["children"].tolist():
        for j in range(_up(lengths[s], ps)):
            refs[tables[s][j]] -= 1
        lengths[s] = 0
    k, v = x["k_pool"].double(), x["v_pool"].double()
    for a, b in copies:
        k[:, b] = k[:, a]
        v[:, b] = v[:, a]
    return {"k_pool": k, "v_pool": v, "tables": _i32(tables), "refs": _i32(refs), "lengths": _i32(lengths)}


def _exact_compact(case, x):
    refs, tables, lengths = x["refs"].tolist(), x["tables"].tolist(), x["lengths"].tolist()
    live = [p for p, c in enumerate(refs) if c > 0]
    n = len(live)
    moved = [p for p in live if p >= n]
    holes = [p for p in range(n) if refs[p] == 0]
    to = {p: p for p in live}
    to.update(zip(moved, holes))
    k, v = x["k_pool"].double(), x["v_pool"].double()
    after = [0] * len(refs)
    for p, q in to.items():
        after[q] = refs[p]
        if p != q:
            k[:, q] = x["k_pool"][:, p].double()
            v[:, q] = x["v_pool"][:, p].double()
    out = x["tables_out"].tolist()
    for s, row in enumerate(tables):
        for j in range(_up(lengths[s], case["page"])):
            out[s][j] = to[row[j]]
    return {"k_pool": k, "v_pool": v, "tables_out": _i32(out), "refs_out": _i32(after),
            "remap": _i32([to.get(p, -1) for p in range(len(refs))]), "counts": _i32([n, len(moved)])}


def exact(case, seed):
    if case["kind"] == "attn" and work(case)["flops"] > 4e12:
        return None
    x = _INPUTS[case["kind"]](case, seed)
    return {"rope": _exact_rope, "attn": _exact_attn, "copy": _exact_copy, "branch": _exact_branch,
            "compact": _exact_compact}[case["kind"]](case, x)
