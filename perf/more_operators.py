"""More operators of a server that keeps many sequences in one paged cache, as measurable cases.

Four operators of one step of such a server, in the order of the step: norms of
queries and keys for each head with the rotary positions and the append to the
pages (`norm_rope_append`), attention in a sliding window with a few first tokens
that stay visible (`sink_attention`), attention of a batch whose sequences share
long prefixes (`shared_attention`), and the log probabilities of given tokens with
entropy and top alternatives from a step's logits (`token_logprobs`).

`run` computes each either through the framework (own) or in plain torch
operations in 32 bits.  Head layouts, page sizes, lengths and the vocabulary are
those of the repository's workloads and tests.
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
EPS = 1e-6       # of the norms
SPARE_PAGES = 4  # pages that no sequence owns


def _storage(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _dtype(case):
    return _storage(case["dtype"] if case["kind"] == "logp" else MODELS[case["model"]][5])


def _esz(case):
    return 2 if _dtype(case) == torch.bfloat16 else 4


# ----------------------------------------------------------------------------- the cases

def _norm(name, model, seqs, new_lo, new_hi, ctx_lo, ctx_hi, lens_seed, layout="half", rotary=0, theta=1e6, far=0,
          page=16, pad=0):
    return {"name": name, "kind": "norm", "model": model, "seqs": seqs, "new_lo": new_lo, "new_hi": new_hi,
            "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "lens_seed": lens_seed, "layout": layout,
            "rotary": rotary or MODELS[model][3], "theta": theta, "far": far, "page": page, "pad": pad}


def _sinks(name, model, seqs, new_lo, new_hi, ctx_lo, ctx_hi, lens_seed, window, sinks, lse=False, page=16, pad=0):
    return {"name": name, "kind": "sinks", "model": model, "seqs": seqs, "new_lo": new_lo, "new_hi": new_hi,
            "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "lens_seed": lens_seed, "window": window, "sinks": sinks, "lse": lse,
            "page": page, "pad": pad}


def _shared(name, model, groups, each, new_lo, new_hi, doc_lo, doc_hi, own_lo, own_hi, lens_seed, alone=0, lse=False,
            page=16, pad=0):
    return {"name": name, "kind": "shared", "model": model, "groups": groups, "each": each, "new_lo": new_lo,
            "new_hi": new_hi, "doc_lo": doc_lo, "doc_hi": doc_hi, "own_lo": own_lo, "own_hi": own_hi,
            "lens_seed": lens_seed, "alone": alone, "lse": lse, "page": page, "pad": pad}


def _logp(name, rows, vocab, dtype, tokens, top, banned=0.0, pad=0):
    return {"name": name, "kind": "logp", "rows": rows, "vocab": vocab, "dtype": dtype, "tokens": tokens, "top": top,
            "banned": banned, "pad": pad}


def listed():
    return [
        # one decoding step of eight short conversations: nothing but latency
        _norm("norm_step15b_8", "qwen15b", 8, 1, 1, 100, 4000, 1),
        # fp32, a few ragged chunks with an idle sequence, interleaved pairs of half the head at far positions
        _norm("norm_f32_ragged", "tiny", 7, 0, 200, 1, 900, 13, layout="interleaved", rotary=32, theta=1e4, far=900000,
              page=8, pad=3),
        # prefill chunks of four long documents
        _norm("norm_chunk7b_16384", "qwen7b", 4, 4096, 4096, 1, 12288, 3),
        # a full server's decoding step of long-running conversations, each in its window and its first tokens
        _sinks("sinks_step7b_64", "qwen7b", 64, 1, 1, 500, 16384, 5, window=4096, sinks=4),
        # chunks of documents that are read in a window, at head size 64
        _sinks("sinks_chunk64_4", "small64", 4, 500, 2048, 300, 4096, 7, window=1024, sinks=16),
        # fp32 storage: ragged drafts and chunks with their log-sums, small pages, padded rows behind
        _sinks("sinks_f32_6", "tiny", 6, 1, 64, 1, 1500, 9, window=200, sinks=4, lse=True, page=8, pad=5),
        # eight answers to one document, all at their next token
        _shared("shared_step15b_8", "qwen15b", 1, 8, 1, 1, 3000, 3000, 1, 60, 4),
        # a full server's decoding step: four long documents, sixteen conversations about each
        _shared("shared_step7b_64", "qwen7b", 4, 16, 1, 1, 4096, 16384, 20, 500, 6),
        # fp32 storage: drafts of a few tokens over three prompts, two conversations without one, log-sums
        _shared("shared_draft_f32_14", "tiny", 3, 4, 1, 6, 200, 1500, 0, 90, 8, alone=2, lse=True, page=8, pad=3),
        # the logits that one decoding step returns: its token, and five alternatives
        _logp("logp_step_1", 1, 152064, "f32", 1, 5),
        # a full server's step: 20 alternatives each, part of the vocabulary ruled out
        _logp("logp_step_64", 64, 152064, "bf16", 1, 20, banned=0.1),
        # a prompt scored token by token
        _logp("logp_score_2048", 2048, 152064, "bf16", 1, 0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(max(hi, 1))))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "step", "draft", "chunk", "f32", "shared", "shared", "shared_draft", "shared_f32",
                       "logp", "logp", "logp_small"])
    page = rng.choice([16, 16, 16, 32, 64, 8, 1])
    seed = rng.randrange(1 << 20)
    big = rng.choice(["qwen15b", "qwen15b", "qwen7b", "small64"])
    if kind == "norm":
        model = rng.choice([big, "tiny", "tiny128"])
        seqs = _log_int(rng, 1, 64)
        hd = MODELS[model][3]
        c = _norm("", model, seqs, rng.choice([0, 1]), _log_int(rng, 1, 8192 // seqs), 1, _log_int(rng, 2, 8192), seed,
                  layout=rng.choice(["half", "interleaved"]), rotary=rng.choice([hd, hd, hd // 2, hd // 4, 48]),
                  theta=rng.choice([1e4, 1e6]), far=rng.choice([0, 0, _log_int(rng, 1000, 1000000)]), page=page,
                  pad=rng.choice([0, 0, 7]))
    elif kind == "step":
        c = _sinks("", big, _log_int(rng, 1, 64), 1, 1, 1, _log_int(rng, 2, 16384), seed, _log_int(rng, 1, 4096),
                   _log_int(rng, 1, 64), lse=rng.random() < 0.3, page=page)
    elif kind == "draft":
        c = _sinks("", big, _log_int(rng, 1, 24), 1, rng.randrange(2, 17), 1, _log_int(rng, 2, 8192), seed,
                   _log_int(rng, 1, 4096), _log_int(rng, 1, 64), lse=rng.random() < 0.3, page=page)
    elif kind == "chunk":
        c = _sinks("", big, _log_int(rng, 1, 4), 100, _log_int(rng, 101, 2048), 1, _log_int(rng, 2, 4096), seed,
                   _log_int(rng, 1, 3000), _log_int(rng, 1, 64), page=page)
    elif kind == "f32":
        c = _sinks("", rng.choice(["tiny", "tiny128"]), _log_int(rng, 1, 16), rng.choice([0, 1]), _log_int(rng, 1, 300),
                   1, _log_int(rng, 2, 3000), seed, _log_int(rng, 1, 1000), _log_int(rng, 1, 64), lse=rng.random() < 0.5,
                   page=page, pad=rng.choice([0, 4]))
    elif kind in ("shared", "shared_draft", "shared_f32"):
        groups = _log_int(rng, 1, 8)
        model = rng.choice(["tiny", "tiny128"]) if kind == "shared_f32" else big
        doc = _log_int(rng, 64, 3000 if kind == "shared_f32" else 16384)
        c = _shared("", model, groups, _log_int(rng, 1, 48 // groups), rng.choice([0, 1]),
                    1 if kind == "shared" else rng.randrange(1, 13), max(1, doc // rng.choice([1, 4, 50])), doc, 0,
                    _log_int(rng, 2, 800), seed, alone=rng.choice([0, 0, 1, 3]), lse=rng.random() < 0.3, page=page,
                    pad=rng.choice([0, 0, 3]))
    else:
        dtype = rng.choice(["f32", "bf16", "bf16"])
        vocab = _log_int(rng, 1000, 152064) if kind == "logp" else _log_int(rng, 40, 2000)
        rows = _log_int(rng, 1, min(2048, (300 if dtype == "bf16" else 150) * 1000000 // vocab))
        c = _logp("", rows, vocab, dtype, rng.choice([1, 1, 1, 0, 4]), rng.choice([0, 1, 5, 20, 32]),
                  banned=rng.choice([0.0, 0.0, 0.3]), pad=rng.choice([0, 0, 8, 3]))
    del c["name"]
    return c


def _up(a, b):
    return -(-a // b)


def _lens(case):
    """New tokens and whole lengths of the case's sequences, and (shared) their documents' lengths, by group."""
    r = random.Random(case["lens_seed"])
    new, total, docs = [], [], []
    if case["kind"] == "shared":
        ps = case["page"]
        for g in range(case["groups"]):
            doc = case["doc_hi"] if g == 0 else _log_int(r, case["doc_lo"], case["doc_hi"])
            docs.append(max(doc // ps, 1) * ps)  # (whole pages are shared)
            for i in range(case["each"]):
                n = case["new_hi"] if i == 0 else _log_int(r, case["new_lo"], case["new_hi"])
                if case["new_lo"] == 0 and i and r.random() < 0.2:
                    n = 0
                new.append(n)
                total.append(docs[-1] + (case["own_hi"] if i == 0 else r.randint(case["own_lo"], case["own_hi"])) + n)
        for _ in range(case["alone"]):  # sequences of no group
            new.append(case["new_hi"])
            total.append(_log_int(r, 1, case["doc_hi"]) + new[-1])
        return new, total, docs
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
    return new, total, docs


def work(case):
    if case["kind"] == "logp":
        n, v, k = case["rows"], case["vocab"], case["tokens"]
        return {"bytes": n * v * _esz(case) + n * (8 + 8 * k + 8 * case["top"]), "flops": 5 * n * v}
    _, nq, nkv, hd, _, _ = MODELS[case["model"]]
    esz = _esz(case)
    new, total, docs = _lens(case)
    rows = sum(new)
    if case["kind"] == "norm":
        return {"bytes": 2 * rows * (nq + 2 * nkv) * hd * esz + 2 * hd * esz,
                "flops": rows * (nq + nkv) * (4 * hd + 3 * case["rotary"])}
    keys = pairs = 0
    for s, (n, t) in enumerate(zip(new, total)):
        if not n:
            continue
        if case["kind"] == "sinks":
            w, first = case["window"], case["sinks"]
            begin = max(0, t - n + 1 - w)  # of the first row's window
            keys += t - begin + min(first, begin)
            pairs += sum(min(p + 1, w) + min(first, max(0, p + 1 - w)) for p in range(t - n, t))
        else:
            g = s // case["each"]
            keys += t - (docs[g] if g < case["groups"] else 0)
            pairs += sum(p + 1 for p in range(t - n, t))
    if case["kind"] == "shared":
        keys += sum(d for g, d in enumerate(docs) if any(new[g * case["each"]:(g + 1) * case["each"]]))
    by = rows * nq * hd * 2 * esz + keys * nkv * hd * 2 * esz + (4 * rows * nq if case["lse"] else 0)
    return {"bytes": by, "flops": 4 * hd * nq * pairs}


# ----------------------------------------------------------------------------- inputs

def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + salt) % (1 << 62))
    return g


def _normal(seed, salt, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=_gen(seed, salt), device="cuda", dtype=torch.float32) * scale).to(dtype)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _batch_inputs(case, seed):
    """A ragged batch: row starts, lengths, block tables over shuffled pages, and the pools of two layers."""
    _, _, nkv, hd, _, _ = MODELS[case["model"]]
    new, total, docs = _lens(case)
    ps = case["page"]
    # a shared document's pages are its group's first pages, held once
    shared = [docs[s // case["each"]] // ps if docs and s // case["each"] < len(docs) else 0 for s in range(len(new))]
    need = [_up(t, ps) for t in total]
    n_pages = sum(need) - sum(shared) + sum(d // ps for d in docs) + SPARE_PAGES
    width = max(max(need), 1)
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(int(seed))).to(torch.int32)
    tables = torch.zeros(len(total), width, dtype=torch.int32)
    at = 0
    of_doc = []
    for d in docs:
        of_doc.append(order[at:at + d // ps])
        at += d // ps
    for s, k in enumerate(need):
        if shared[s]:
            tables[s, :shared[s]] = of_doc[s // case["each"]]
        tables[s, shared[s]:k] = order[at:at + k - shared[s]]
        at += k - shared[s]
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    shape = (2, n_pages, nkv, ps, hd)
    dt = _dtype(case)
    return {"rows": starts[-1], "n_rows": starts[-1] + case["pad"], "most_new": max(max(new), 1),
            "row_start": _i32(starts), "length": _i32(total), "tables": tables.cuda(),
            "k_pool": _normal(seed, 1, shape, dt), "v_pool": _normal(seed, 2, shape, dt), "layer": 1}


def _norm_inputs(case, seed):
    _, nq, nkv, hd, _, _ = MODELS[case["model"]]
    x = _batch_inputs(case, seed)
    n, dt = x["n_rows"], _dtype(case)
    # the rows of a fused projection, of which q, k and v are slices; heads of different sizes, as projections have
    size = torch.exp(_normal(seed, 4, (nq + 2 * nkv, 1), torch.float32))
    qkv = (_normal(seed, 3, (max(n, 1), nq + 2 * nkv, hd), torch.float32) * size).to(dt).view(max(n, 1), -1)[:n]
    x["q"] = qkv[:, :nq * hd].view(n, nq, hd)
    x["k"] = qkv[:, nq * hd:(nq + nkv) * hd].view(n, nkv, hd)
    x["v"] = qkv[:, (nq + nkv) * hd:].view(n, nkv, hd)
    x["q_norm"] = (1.0 + 0.2 * _normal(seed, 5, (hd,), torch.float32)).to(dt)
    x["k_norm"] = (1.0 + 0.2 * _normal(seed, 6, (hd,), torch.float32)).to(dt)
    x["q_out"] = torch.zeros(n, nq, hd, dtype=dt, device="cuda")
    # explicit rotary positions where the sequence continues one whose head is no longer cached
    x["positions"] = (torch.arange(n, dtype=torch.int32, device="cuda") + case["far"]) if case["far"] else None
    return x


def _attn_inputs(case, seed):
    _, nq, _, hd, _, _ = MODELS[case["model"]]
    x = _batch_inputs(case, seed)
    n = x["n_rows"]
    x["q"] = _normal(seed, 3, (n, nq, hd), _dtype(case), 2.0)
    x["out"] = torch.zeros(n, nq, hd, dtype=_dtype(case), device="cuda")
    x["lse"] = torch.zeros(n, nq, dtype=torch.float32, device="cuda") if case["lse"] else None
    if case["kind"] == "shared":
        _, _, docs = _lens(case)
        x["seq_start"] = _i32([g * case["each"] for g in range(case["groups"] + 1)])
        x["shared_len"] = _i32(docs)
    return x


def _logp_inputs(case, seed):
    n, v = case["rows"], case["vocab"]
    dt = _dtype(case)
    logits = torch.empty(n, v + case["pad"], dtype=dt, device="cuda")[:, :v]
    g = _gen(seed, 1)
    # a model's logits: a broad bulk, and a few likely tokens far above it
    likely = torch.randperm(v, generator=g, device="cuda")[:min(v, 40)]
    for a in range(0, n, 256):
        b = min(n, a + 256)
        z = torch.randn((b - a, v), generator=g, device="cuda").mul_(2.0)
        z[:, likely] += torch.rand((b - a, likely.numel()), generator=g, device="cuda") * 14.0
        if case["banned"]:
            z.masked_fill_(torch.rand((b - a, v), generator=g, device="cuda") < case["banned"], -math.inf)
        logits[a:b] = z
    # likely tokens mostly, some others, and rows without one (padding)
    t = likely[torch.randint(likely.numel(), (n, case["tokens"]), generator=g, device="cuda")]
    other = torch.randint(v, t.shape, generator=g, device="cuda")
    pick = torch.rand(t.shape, generator=g, device="cuda")
    tokens = torch.where(pick < 0.7, t, torch.where(pick < 0.95, other, -1)).to(torch.int32)
    f = dict(dtype=torch.float32, device="cuda")
    return {"logits": logits, "tokens": tokens if case["tokens"] else None,
            "logprob": torch.zeros(tokens.shape, **f) if case["tokens"] else None,
            "entropy": torch.zeros(n, **f), "lse": torch.zeros(n, **f),
            "top_token": torch.zeros(n, case["top"], dtype=torch.int32, device="cuda") if case["top"] else None,
            "top_logprob": torch.zeros(n, case["top"], **f) if case["top"] else None}


_INPUTS = {"norm": _norm_inputs, "sinks": _attn_inputs, "shared": _attn_inputs, "logp": _logp_inputs}


def prepare(case, seed):
    x = _INPUTS[case["kind"]](case, seed)
    x["case"] = dict(case)
    if own:  # the handles that a server keeps: the context and the descriptors of its buffers
        _handles(case, x)
    return x


# ----------------------------------------------------------------------------- the framework's calls

def _handles(case, x):
    import paper_2609_30884_amd as crf
    x["crf"] = crf
    if case["kind"] == "logp":
        d, nq, nkv, hd, f, dt = MODELS["qwen15b"]
        x["ctx"] = crf.Context(crf.make_dims(2, d, nq, nkv, hd, f, dtype=dt), 1, 0)
        return
    d, nq, nkv, hd, f, dt = MODELS[case["model"]]
    x["ctx"] = crf.Context(crf.make_dims(2, d, nq, nkv, hd, f, rms_eps=EPS, dtype=dt), 1, 0)
    x["pool"] = crf.page_pool(x["k_pool"], x["v_pool"], case["page"])
    x["batch"] = crf.seq_batch(x["row_start"], x["length"], x["tables"], x["n_rows"], x["most_new"])
    if case["kind"] == "norm":
        x["rope"] = crf.rope(case["rotary"], case["theta"], layout=case["layout"])
    if case["kind"] == "shared":
        x["groups"] = crf.seq_groups(x["seq_start"], x["shared_len"])


def _run_own(x):
    crf, case = x["crf"], x["case"]
    kind = case["kind"]
    if kind == "norm":
        crf.norm_rope_append(x["ctx"], x["rope"], x["batch"], x["q"], x["k"], x["v"], x["q_norm"], x["k_norm"],
                             x["pool"], x["layer"], x["q_out"], x["positions"])
    elif kind == "sinks":
        crf.sink_attention(x["ctx"], x["batch"], x["q"], x["pool"], x["layer"], x["out"], case["window"], case["sinks"],
                           lse=x["lse"])
    elif kind == "shared":
        crf.shared_attention(x["ctx"], x["batch"], x["groups"], x["q"], x["pool"], x["layer"], x["out"], lse=x["lse"])
    else:
        crf.token_logprobs(x["ctx"], x["logits"], x["tokens"], x["logprob"], entropy=x["entropy"], lse=x["lse"],
                           top_token=x["top_token"], top_logprob=x["top_logprob"])


# ----------------------------------------------------------------------------- the plain forms

def _rows_of(x):
    """Sequence and position of each row."""
    row = torch.arange(x["rows"], device="cuda")
    start = x["row_start"].long()
    seq = (row[:, None] >= start[None, 1:]).sum(1)
    return seq, x["length"].long()[seq] - start[seq + 1] + row


def _normed(t, gain):
    t = t.float()
    return t * (t.square().mean(-1, keepdim=True) + EPS).rsqrt() * gain.float()


def _rotate(t, cos, sin, r, layout):
    a, b = (t[..., 0:r:2], t[..., 1:r:2]) if layout == "interleaved" else (t[..., :r // 2], t[..., r // 2:r])
    x, y = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((x, y), -1).flatten(-2) if layout == "interleaved" else torch.cat((x, y), -1)
    return torch.cat((turned, t[..., r:]), -1)


def _plain_norm(x):
    case, n = x["case"], x["rows"]
    seq, pos = _rows_of(x)
    r = case["rotary"]
    f = torch.arange(0, r, 2, dtype=torch.float64, device="cuda").div(-r).mul(math.log(case["theta"])).exp()
    angle = (pos if x["positions"] is None else x["positions"][:n]).double()[:, None] * f
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x["q_out"][:n] = _rotate(_normed(x["q"][:n], x["q_norm"]), cos, sin, r, case["layout"]).to(x["q"].dtype)
    k = _rotate(_normed(x["k"][:n], x["k_norm"]), cos, sin, r, case["layout"]).to(x["k"].dtype)
    page, slot = x["tables"][seq, pos // case["page"]].long(), pos % case["page"]
    x["k_pool"][x["layer"]][page, :, slot] = k
    x["v_pool"][x["layer"]][page, :, slot] = x["v"][:n]


def _plain_attn(x):
    """The batch padded to its longest sequence: scores, softmax and products in 32 bits."""
    case, n = x["case"], x["rows"]
    ps = case["page"]
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
    if case["kind"] == "sinks":
        hide |= (j <= p[..., None] - case["window"]) & (j >= case["sinks"])
    s.masked_fill_(hide[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    s.sub_(top).exp_()
    z = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(seqs, nkv, g * most, keys), v).view(seqs, nkv, g, most, hd) / z
    x["out"][:n] = o.permute(0, 3, 1, 2, 4).reshape(seqs, most, nq, hd)[seq, at].to(x["out"].dtype)
    if x["lse"] is not None:
        lse = (top + z.log()).squeeze(-1)
        x["lse"][:n] = lse.permute(0, 3, 1, 2).reshape(seqs, most, nq)[seq, at]


def _plain_logp(x):
    z = x["logits"].float()
    m = z.amax(1, keepdim=True)
    d = z - m
    e = d.exp()
    total = e.sum(1, keepdim=True)
    x["lse"].copy_((m + total.log()).squeeze(1))
    x["entropy"].copy_((total.log() - torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / total).squeeze(1))
    if x["tokens"] is not None:
        t = x["tokens"].long()
        lp = d.gather(1, t.clamp(min=0)) - total.log()
        x["logprob"].copy_(torch.where(t < 0, 0.0, lp))
    if x["top_token"] is not None:
        # unique keys in the order of the values, the lowest index first among equals
        v = z.shape[1]
        b = (z + 0.0).view(torch.int32).long()
        key = (torch.where(b < 0, b ^ 0x7fffffff, b) << 32) + (v - 1 - torch.arange(v, device="cuda"))
        for i in range(x["top_token"].shape[1]):
            best = key.amax(1, keepdim=True)
            at = v - 1 - (best & 0xffffffff)
            x["top_token"][:, i] = at.squeeze(1).int()
            x["top_logprob"][:, i] = (d.gather(1, at) - total.log()).squeeze(1)
            key.scatter_(1, at, -(1 << 63))


_PLAIN = {"norm": _plain_norm, "sinks": _plain_attn, "shared": _plain_attn, "logp": _plain_logp}
_OUTPUTS = {"norm": ("q_out", "k_pool", "v_pool"), "sinks": ("out", "lse"), "shared": ("out", "lse"),
            "logp": ("logprob", "entropy", "lse", "top_token", "top_logprob")}


def run(state):
    kind = state["case"]["kind"]
    if own:
        _run_own(state)
    else:
        _PLAIN[kind](state)
    return {name: state[name] for name in _OUTPUTS[kind]}


# ----------------------------------------------------------------------------- from the definitions, in 64 bits

def _exact_norm(case, x):
    """Each pair of a normed head as a complex number times e^(i angle), sequence by sequence."""
    new, total, _ = _lens(case)
    half = case["rotary"] // 2
    freq = torch.tensor([case["theta"] ** (-2.0 * i / case["rotary"]) for i in range(half)], dtype=torch.float64,
                        device="cuda")
    inter = case["layout"] == "interleaved"
    first = torch.arange(half, device="cuda") * (2 if inter else 1)
    second = first + (1 if inter else half)

    def turn(t, gain, pos):
        t = t.double()
        t = t / torch.sqrt((t * t).sum(-1, keepdim=True) / t.shape[-1] + EPS) * gain.double()
        a = pos[:, None] * freq
        z = torch.complex(t[..., first], t[..., second]) * torch.polar(torch.ones_like(a), a)[:, None]
        t[..., first], t[..., second] = z.real, z.imag
        return t

    q_out, kp, vp = x["q_out"].double(), x["k_pool"].double(), x["v_pool"].double()
    row = 0
    for i, (n, t) in enumerate(zip(new, total)):
        if not n:
            continue
        p = torch.arange(t - n, t, device="cuda")
        angle_at = p.double() if not case["far"] else torch.arange(row, row + n, device="cuda").double() + case["far"]
        q_out[row:row + n] = turn(x["q"][row:row + n], x["q_norm"], angle_at)
        page = x["tables"][i].long()[torch.div(p, case["page"], rounding_mode="floor")]
        kp[x["layer"], page, :, p % case["page"]] = turn(x["k"][row:row + n], x["k_norm"], angle_at)
        vp[x["layer"], page, :, p % case["page"]] = x["v"][row:row + n].double()
        row += n
    return {"q_out": q_out, "k_pool": kp, "v_pool": vp}


def _exact_attn(case, x):
    """One sequence, K/V head and block of queries at a time."""
    new, total, _ = _lens(case)
    nq, hd = x["q"].shape[1:]
    nkv = x["k_pool"].shape[2]
    g = nq // nkv
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
                seen = key <= p
                if case["kind"] == "sinks":
                    seen = seen & ((key > p - case["window"]) | (key < case["sinks"]))
                s = torch.where(seen, s, torch.full_like(s, -math.inf))
                out[row + b:row + e, h * g:(h + 1) * g] = (torch.softmax(s, -1).view(-1, t) @ v).view(e - b, g, hd)
                if lse is not None:
                    lse[row + b:row + e, h * g:(h + 1) * g] = torch.logsumexp(s, -1)
        row += n
    return {"out": out, "lse": lse}


def _exact_logp(case, x):
    """Row blocks: probabilities, their entropy as a sum over p, and the values sorted."""
    n, k = case["rows"], case["top"]
    d = dict(dtype=torch.float64, device="cuda")
    out = {"logprob": torch.zeros(n, case["tokens"], **d) if case["tokens"] else None, "entropy": torch.zeros(n, **d),
           "lse": torch.zeros(n, **d), "top_token": _i32([[0] * k] * n) if k else None,
           "top_logprob": torch.zeros(n, k, **d) if k else None}
    for a in range(0, n, 64):
        z = x["logits"][a:a + 64].double()
        lse = torch.logsumexp(z, 1, keepdim=True)
        log_p = z - lse
        p = torch.exp(log_p)
        out["lse"][a:a + 64] = lse[:, 0]
        out["entropy"][a:a + 64] = -torch.where(p > 0, p * log_p, torch.zeros_like(p)).sum(1)
        if case["tokens"]:
            t = x["tokens"][a:a + 64].long()
            out["logprob"][a:a + 64] = torch.where(t >= 0, log_p.gather(1, t.clamp(min=0)), torch.zeros_like(log_p[:, :1]))
        if k:
            value, at = torch.sort(z, dim=1, descending=True, stable=True)
            out["top_token"][a:a + 64] = at[:, :k].int()
            out["top_logprob"][a:a + 64] = value[:, :k] - lse
    return out


def exact(case, seed):
    if case["kind"] in ("sinks", "shared") and work(case)["flops"] > 4e12:
        return None
    x = _INPUTS[case["kind"]](case, seed)
    return {"norm": _exact_norm, "sinks": _exact_attn, "shared": _exact_attn, "logp": _exact_logp}[case["kind"]](case, x)
