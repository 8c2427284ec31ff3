"""The operators of a verification step over drafted tokens (and of the training that goes with it), as cases to measure.

A serving step that checks drafted tokens runs, per step,  plan_pages (which cache rows the new tokens take),  per layer
qk_norm_rope (heads normed and rotated, K / V rows into the cache) and tree_attention (every drafted token against the
cache and its own ancestors), and at the end token_logprobs (what the model says about the drafted tokens).  The gradients
of the first and the last of these that have any (qk_norm_rope, token_logprobs) belong to the training side.

`own` false: the plain form of each operator in elementary torch operations.  `own` true: this package's kernels."""
import math
import random

import torch

own = False

PAGE = 128          # cache rows of a page
THETA = 500000.0    # rotary base of the 8B / 70B shapes
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a small decode batch takes its next cache rows: a handful of numbers, latency alone
        {"name": "plan 8 sequences", "op": "plan", "seqs": 8, "new_hi": 8, "past_hi": 4096, "scarce": False, "lens": 1},
        # a large serving batch with prompt chunks among single tokens, block tables for 131072 positions each
        {"name": "plan 1024 sequences", "op": "plan", "seqs": 1024, "new_hi": 64, "past_hi": 131072, "scarce": False, "lens": 2},
        # one layer of a verification step of 8 sequences with about 12 drafted tokens each, into the FP8 cache
        {"name": "rope 96 tokens fp8 cache", "op": "rope", "tokens": 96, "n_kv": 8, "rep": 4, "hd": 128, "gains": True, "type": "bf16", "cache": "fp8"},
        # one layer of a long prompt chunk, into pages in the model's type
        {"name": "rope 16411 tokens", "op": "rope", "tokens": 16411, "n_kv": 8, "rep": 4, "hd": 128, "gains": True, "type": "bf16", "cache": "same"},
        # the gradient of the same for a training batch
        {"name": "rope gradient 8195 tokens", "op": "rope_bwd", "tokens": 8195, "n_kv": 8, "rep": 4, "hd": 128, "gains": True, "type": "bf16"},
        # one sequence decoding one token over a short cache: latency alone
        {"name": "tree 1 token over 700", "op": "tree", "seqs": 1, "new_lo": 1, "new_hi": 1, "kv_lo": 700, "kv_hi": 700, "n_kv": 8, "rep": 4, "hd": 128,
         "type": "bf16", "cache": "same", "tree": False, "paged": True, "lens": 3},
        # a verification batch: ordinary trees over ordinary contexts
        {"name": "tree 16 x 32 over 8192", "op": "tree", "seqs": 16, "new_lo": 9, "new_hi": 32, "kv_lo": 2048, "kv_hi": 8192, "n_kv": 8, "rep": 4, "hd": 128,
         "type": "bf16", "cache": "same", "tree": True, "paged": True, "lens": 4},
        # two long documents, the widest trees, the head counts of the 70B shape: the most work
        {"name": "tree 2 x 64 over 131072", "op": "tree", "seqs": 2, "new_lo": 64, "new_hi": 64, "kv_lo": 100000, "kv_hi": 131072, "n_kv": 8, "rep": 8, "hd": 128,
         "type": "bf16", "cache": "same", "tree": True, "paged": True, "lens": 5},
        # many sequences with short drafts over the FP8 cache
        {"name": "tree 24 x 8 over 10000 fp8", "op": "tree", "seqs": 24, "new_lo": 1, "new_hi": 8, "kv_lo": 3001, "kv_hi": 10000, "n_kv": 8, "rep": 4, "hd": 128,
         "type": "bf16", "cache": "fp8", "tree": True, "paged": True, "lens": 6},
        # the logits of a few drafted tokens, with alternatives
        {"name": "logprobs 33 rows", "op": "logprobs", "rows": 33, "vocab": 128256, "type": "f32", "top": 8, "temperature": 1.0, "padded": False},
        # scoring a prompt or a training batch
        {"name": "logprobs 4096 rows", "op": "logprobs", "rows": 4096, "vocab": 128256, "type": "bf16", "top": 5, "temperature": 1.0, "padded": False},
        # the gradient with respect to the logits, entropy term included
        {"name": "logprobs gradient 2048 rows", "op": "logprobs_bwd", "rows": 2048, "vocab": 128256, "type": "bf16", "temperature": 1.0, "padded": False},
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(("plan", "rope", "rope", "rope_bwd", "tree", "tree", "tree", "logprobs", "logprobs", "logprobs_bwd"))
    if op == "plan":
        seqs = _log(rng, 1, 1024)
        return {"op": op, "seqs": seqs, "new_hi": _log(rng, 1, min(4096, 65536 // seqs)), "past_hi": _log(rng, 1, 131072), "scarce": rng.random() < 0.25,
                "lens": rng.randrange(1 << 20)}
    heads = {"n_kv": rng.choice((1, 2, 4, 8)), "rep": rng.choice((1, 2, 3, 4, 5, 7, 8)), "hd": rng.choice((64, 128, 128))}
    if op == "rope":
        cache = rng.choice(("same", "same", "fp8"))
        heads["rep"] = min(heads["rep"], 4 if heads["n_kv"] == 8 else 8)
        return {"op": op, "tokens": _log(rng, 1, 4096 if cache == "fp8" else 16411), **heads, "gains": rng.random() < 0.7, "type": rng.choice(("bf16", "bf16", "f16")),
                "cache": cache}
    if op == "rope_bwd":
        heads["rep"] = min(heads["rep"], 4 if heads["n_kv"] == 8 else 8)
        return {"op": op, "tokens": _log(rng, 1, 8195), **heads, "gains": rng.random() < 0.8, "type": rng.choice(("bf16", "bf16", "f16"))}
    if op == "tree":
        seqs = _log(rng, 1, 32)
        new_hi = _log(rng, 1, 64)
        kv_hi = _log(rng, new_hi, 262144 // max(seqs, 2))
        return {"op": op, "seqs": seqs, "new_lo": rng.randint(1, new_hi), "new_hi": new_hi, "kv_lo": rng.randint(max(new_hi, kv_hi // 4), kv_hi), "kv_hi": kv_hi,
                **heads, "type": rng.choice(("bf16", "bf16", "f16")), "cache": rng.choice(("same", "same", "fp8")), "tree": rng.random() < 0.7,
                "paged": rng.random() < 0.7, "lens": rng.randrange(1 << 20)}
    vocab = _log(rng, 1000, 160000)
    rows = _log(rng, 1, min(4096, 4096 * 128256 // vocab))
    kind = rng.choice(("f32", "bf16", "bf16", "f16"))
    if op == "logprobs_bwd":
        rows = min(rows, 2048)
        if kind == "f32":
            rows = min(rows, 1024)
        return {"op": op, "rows": rows, "vocab": vocab, "type": kind, "temperature": rng.choice((1.0, 0.7, 2.0)), "padded": rng.random() < 0.3}
    if kind == "f32":
        rows = min(rows, 2048)
    return {"op": op, "rows": rows, "vocab": vocab, "type": kind, "top": rng.choice((0, 1, 5, 8, 20)), "temperature": rng.choice((1.0, 0.7, 2.0)),
            "padded": rng.random() < 0.3}


def _plan_lengths(case):
    """(past, new, owned pages, pages on the free list) of every sequence: a function of the case alone."""
    r = random.Random(case["lens"])
    past = [r.randint(0, case["past_hi"]) for _ in range(case["seqs"])]
    new = [r.randint(0, case["new_hi"]) if r.random() < 0.5 else min(1, case["new_hi"]) for _ in range(case["seqs"])]
    # what a sequence holds already covers its past; after a rejected draft some hold a page more
    owned = [-(-p // PAGE) + (1 if r.random() < 0.2 else 0) for p in past]
    need = sum(max(0, -(-(p + n) // PAGE) - o) for p, n, o in zip(past, new, owned))
    free = need // 2 if case["scarce"] else need + 37
    return past, new, owned, free


def _max_blocks(case):
    return -(-(case["past_hi"] + case["new_hi"]) // PAGE) + 2


def _tree_lengths(case):
    r = random.Random(case["lens"])
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    kv = [r.randint(case["kv_lo"], case["kv_hi"]) for _ in range(case["seqs"])]
    new[0], kv[0] = case["new_hi"], case["kv_hi"]
    return [k - n for k, n in zip(kv, new)], new


def _size(kind):
    return torch.finfo(TYPES[kind]).bits // 8


def work(case):
    op = case["op"]
    if op == "plan":
        past, new, owned, free = _plan_lengths(case)
        taken = min(free, sum(max(0, -(-(p + n) // PAGE) - o) for p, n, o in zip(past, new, owned)))
        # lengths, the table's used entries and the taken pages in; the new table whole, offsets, row and position of every token out
        return {"bytes": 4 * (4 * case["seqs"] + sum(owned) + taken + case["seqs"] * _max_blocks(case) + case["seqs"] + 2 * sum(new)), "flops": 0}
    if op in ("rope", "rope_bwd"):
        t, hd, n_kv = case["tokens"], case["hd"], case["n_kv"]
        n_q, es = n_kv * case["rep"], _size(case["type"])
        table = 4 * hd
        if op == "rope":
            stored = 2 * n_kv * hd * (1 if case["cache"] == "fp8" else es) + (8 if case["cache"] == "fp8" else 0)
            return {"bytes": t * ((n_q + 2 * n_kv) * hd * es + n_q * hd * es + stored + table + 8), "flops": 10 * t * (n_q + n_kv) * hd}
        return {"bytes": t * ((n_q + n_kv) * hd * es * 3 + table + 4), "flops": 20 * t * (n_q + n_kv) * hd}
    if op == "tree":
        past, new = _tree_lengths(case)
        hd, n_kv = case["hd"], case["n_kv"]
        n_q, es = n_kv * case["rep"], _size(case["type"])
        row = 2 * n_kv * hd * (1 if case["cache"] == "fp8" else es) + (8 if case["cache"] == "fp8" else 0)
        kv = sum(past) + sum(new)
        return {"bytes": kv * row + sum(new) * n_q * (hd * es * 2 + 4) + 4 * sum(new) * (-(-case["new_hi"] // 32)),
                "flops": sum(4 * n * (p + n) * n_q * hd for p, n in zip(past, new))}
    n = case["rows"] * case["vocab"]
    if op == "logprobs":
        return {"bytes": n * _size(case["type"]) + case["rows"] * (16 + 8 * case["top"]), "flops": 5 * n}
    return {"bytes": 2 * n * _size(case["type"]) + case["rows"] * 20, "flops": 6 * n}


# ---------------------------------------------------------------------------------------------------------- inputs
def _gen(seed, salt=0):
    return torch.Generator(device="cuda").manual_seed(seed * 1000003 + salt)


def _randn(shape, g, scale=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _rope_tables(positions, hd):
    """cos and sin of position * theta^(-2 i / hd) for every position below `positions`, angles in 64 bits."""
    inv = THETA ** (-torch.arange(0, hd, 2, dtype=torch.float64, device="cuda") / hd)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * inv
    return a.cos().float(), a.sin().float()


def _codes(shape, g):
    """e4m3 codes of rows as a per-row scale leaves them: normal values up to 448."""
    x = torch.randn(shape, generator=g, device="cuda") * 120.0
    return x.clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def prepare(case, seed):
    op, g = case["op"], _gen(seed)
    s = {"case": case, "op": op}
    if op == "plan":
        past, new, owned, free = _plan_lengths(case)
        mb = _max_blocks(case)
        pages = torch.randperm(sum(owned) + free, generator=g, device="cuda").to(torch.int32)
        table = torch.full((case["seqs"], mb), -1, dtype=torch.int32, device="cuda")
        held = torch.arange(mb, device="cuda")[None] < _ints(owned)[:, None]
        table[held] = pages[: sum(owned)]
        s.update(past=_ints(past), new=_ints(new), owned=_ints(owned), table=table, free=pages[sum(owned):].contiguous(), n_free=_ints([free]), total=sum(new))
        s["out"] = {"block_table": torch.empty_like(table), "n_owned": torch.empty_like(s["owned"]), "n_free": torch.empty_like(s["n_free"]),
                    "cu_new": torch.empty(case["seqs"] + 1, dtype=torch.int32, device="cuda"),
                    "slot_map": torch.empty(sum(new), dtype=torch.int32, device="cuda"),
                    "positions": torch.empty(sum(new), dtype=torch.int32, device="cuda"),
                    "info": torch.empty(4, dtype=torch.int32, device="cuda")}
        return s
    if op in ("rope", "rope_bwd"):
        t, hd, n_kv, dt = case["tokens"], case["hd"], case["n_kv"], TYPES[case["type"]]
        n_q = n_kv * case["rep"]
        max_pos = 131072
        cos, sin = _rope_tables(max_pos, hd)
        # what the projection of a layer leaves: one row [queries | keys | values] per token
        qkv = _randn((t, (n_q + 2 * n_kv) * hd), g, 1.5, dt)
        q = qkv[:, : n_q * hd].view(t, n_q, hd)
        k = qkv[:, n_q * hd: (n_q + n_kv) * hd].view(t, n_kv, hd)
        v = qkv[:, (n_q + n_kv) * hd:].view(t, n_kv, hd)
        positions = torch.randint(0, max_pos, (t,), generator=g, device="cuda", dtype=torch.int32)
        s.update(q=q, k=k, v=v, cos=cos, sin=sin, positions=positions, q_gain=None, k_gain=None)
        if case["gains"]:
            s["q_gain"], s["k_gain"] = (1.0 + _randn((hd,), g, 0.25)).to(dt), (1.0 + _randn((hd,), g, 0.25)).to(dt)
        if op == "rope_bwd":
            s.update(dq=_randn((t, n_q, hd), g, 0.02, dt), dk=_randn((t, n_kv, hd), g, 0.02, dt))
            s["out"] = (torch.empty_like(s["dq"]), torch.empty_like(s["dk"]))
            return s
        rows = -(-t // PAGE) * PAGE + PAGE
        s["slots"] = torch.randperm(rows, generator=g, device="cuda")[:t].to(torch.int32)
        s["q_out"] = torch.empty((t, n_q, hd), dtype=dt, device="cuda")
        if case["cache"] == "fp8":
            s.update(k_cache=_codes((rows, n_kv, hd), g), v_cache=_codes((rows, n_kv, hd), g), k_scale=torch.rand(rows, generator=g, device="cuda") + 0.01,
                     v_scale=torch.rand(rows, generator=g, device="cuda") + 0.01)
        else:
            s.update(k_cache=_randn((rows, n_kv, hd), g, 1.0, dt), v_cache=_randn((rows, n_kv, hd), g, 1.0, dt), k_scale=None, v_scale=None)
        return s
    if op == "tree":
        past, new = _tree_lengths(case)
        hd, n_kv, dt = case["hd"], case["n_kv"], TYPES[case["type"]]
        n_q = n_kv * case["rep"]
        total, host = sum(new), random.Random(seed)
        pages = [-(-(p + n) // PAGE) for p, n in zip(past, new)]
        rows = (sum(pages) + 3) * PAGE
        if case["paged"]:
            order = torch.randperm(rows // PAGE, generator=g, device="cuda").to(torch.int32)
            table = torch.full((case["seqs"], max(pages)), -1, dtype=torch.int32, device="cuda")
            table[torch.arange(max(pages), device="cuda")[None] < _ints(pages)[:, None]] = order[: sum(pages)]
            s.update(table=table, row0=None)
        else:
            at, row0 = host.randint(0, PAGE), []
            for p in pages:
                row0.append(at)
                at += p * PAGE
            s.update(table=None, row0=_ints(row0))
        s["q"] = _randn((total, n_q, hd), g, 1.5, dt)
        if case["cache"] == "fp8":
            s.update(k_cache=_codes((rows, n_kv, hd), g), v_cache=_codes((rows, n_kv, hd), g),
                     k_scale=(torch.rand(rows, generator=g, device="cuda") + 0.5) / 120.0, v_scale=(torch.rand(rows, generator=g, device="cuda") + 0.5) / 120.0)
        else:
            s.update(k_cache=_randn((rows, n_kv, hd), g, 1.0, dt), v_cache=_randn((rows, n_kv, hd), g, 1.0, dt), k_scale=None, v_scale=None)
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        s.update(past=_ints(past), cu=_ints(cu), max_new=max(new), max_kv=max(p + n for p, n in zip(past, new)), mask=None)
        if case["tree"]:
            # node i hangs on an earlier node (or on the last committed token) and sees its ancestors and itself
            words, bits = -(-max(new) // 32), []
            for n in new:
                seen = []
                for i in range(n):
                    parent = host.randint(-1, i - 1) if i else -1
                    seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
                bits += [[(m >> (32 * w)) & 0xFFFFFFFF for w in range(words)] for m in seen]
            s["mask"] = torch.tensor(bits, dtype=torch.int64).to("cuda").to(torch.int32).contiguous()
        s["out"] = torch.empty((total, n_q, hd), dtype=dt, device="cuda")
        s["lse"] = torch.empty((total, n_q), dtype=torch.float32, device="cuda")
        return s
    rows, vocab, dt = case["rows"], case["vocab"], TYPES[case["type"]]
    # a vocabulary padded for the projection's tiles leaves rows that are longer than what counts
    width = -(-vocab // 128) * 128 + 128 if case["padded"] else vocab
    logits = torch.empty((rows, width), dtype=dt, device="cuda")
    logits.normal_(0.0, 2.5, generator=g)
    s["logits"] = logits[:, :vocab]
    s["targets"] = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    s["targets"][torch.rand(rows, generator=g, device="cuda") < 0.05] = -1      # positions without a target
    if op == "logprobs_bwd":
        lse, entropy = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        for r in range(0, rows, 256):
            z = s["logits"][r: r + 256].double() / case["temperature"]
            l = z.logsumexp(1)
            lse[r: r + 256] = l
            entropy[r: r + 256] = l - ((z - l[:, None]).exp() * z).sum(1)
        s.update(lse=lse, entropy=entropy, g_logprob=_randn((rows,), g), g_entropy=_randn((rows,), g, 0.1))
        s["out"] = torch.empty((rows, vocab), dtype=dt, device="cuda")
        return s
    f = lambda *shape: torch.empty(shape, dtype=torch.float32, device="cuda")  # noqa: E731
    s["out"] = {"logprob": f(rows), "entropy": f(rows), "lse": f(rows), "top_ids": torch.empty((rows, case["top"]), dtype=torch.int32, device="cuda"),
                "top_logprobs": f(rows, case["top"])}
    return s


# ----------------------------------------------------------------------------------------------------- plain forms
def _plan(s):
    past, new, owned, table = s["past"].long(), s["new"].long(), s["owned"].long(), s["table"]
    seqs, mb = table.shape
    cu = torch.cat([new.new_zeros(1), new.cumsum(0)])
    need = ((past + new + PAGE - 1) // PAGE - owned).clamp(min=0)
    first = need.cumsum(0) - need
    n_free = s["n_free"].long()
    j = torch.arange(mb, device="cuda")[None]
    rank = first[:, None] + j - owned[:, None]          # the how manieth page of this call entry j would take
    fresh = (j >= owned[:, None]) & (j < (owned + need)[:, None]) & (rank < n_free)
    page = s["free"][(n_free - 1 - rank).clamp(0, max(0, s["free"].numel() - 1))] if s["free"].numel() else torch.full_like(table, -1)
    out = torch.where(j < owned[:, None], table, torch.where(fresh, page, torch.full_like(table, -1)))
    granted = fresh.sum(1)
    b = torch.repeat_interleave(torch.arange(seqs, device="cuda"), new, output_size=s["total"])
    pos = past[b] + torch.arange(s["total"], device="cuda") - cu[b]
    held = out[b, pos // PAGE]
    slot = torch.where(held >= 0, held * PAGE + pos % PAGE, torch.full_like(held, -1))
    info = torch.stack([cu[-1], granted.sum(), need.sum() - granted.sum(), (past + new).max()])
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return {"block_table": out, "n_owned": i32(owned + granted), "n_free": i32(n_free - granted.sum()), "cu_new": i32(cu), "slot_map": i32(slot),
            "positions": i32(pos), "info": i32(info)}


def _rotate(x, c, n):
    """Rotation of the pairs (i, i + hd/2); `n` is the sine, or its negative for the inverse."""
    a, b = x.chunk(2, -1)
    return torch.cat([a * c - b * n, b * c + a * n], -1)


def _head_norm(x, gain):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.float() if gain is not None else x


def _rope(s):
    c, n = s["cos"][s["positions"].long()][:, None], s["sin"][s["positions"].long()][:, None]
    q = _rotate(_head_norm(s["q"].float(), s["q_gain"]), c, n).to(s["q"].dtype)
    k = _rotate(_head_norm(s["k"].float(), s["k_gain"]), c, n)
    rows = s["slots"].long()
    if s["k_scale"] is None:
        s["k_cache"][rows], s["v_cache"][rows] = k.to(s["k"].dtype), s["v"]
        return q, s["k_cache"], s["v_cache"]
    v = s["v"].float()
    ks, vs = k.abs().amax((1, 2)).clamp(min=2.0 ** -64) / 448.0, v.abs().amax((1, 2)).clamp(min=2.0 ** -64) / 448.0
    s["k_cache"][rows] = (k / ks[:, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    s["v_cache"][rows] = (v / vs[:, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    s["k_scale"][rows], s["v_scale"][rows] = ks, vs
    return q, s["k_cache"].view(torch.float8_e4m3fn), s["v_cache"].view(torch.float8_e4m3fn), s["k_scale"], s["v_scale"]


def _head_norm_bwd(x, dy, gain, c, n):
    """Gradients of rotate(norm(x) * gain) with respect to x and the gain."""
    dz = _rotate(dy.float(), c, -n)
    if gain is None:
        return dz.to(x.dtype), None
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    xh = x * r
    dg = (dz * xh).sum((0, 1))
    dh = dz * gain.float()
    return (r * (dh - xh * (dh * xh).mean(-1, keepdim=True))).to(dy.dtype), dg


def _rope_bwd(s):
    c, n = s["cos"][s["positions"].long()][:, None], s["sin"][s["positions"].long()][:, None]
    dq, dgq = _head_norm_bwd(s["q"], s["dq"], s["q_gain"], c, n)
    dk, dgk = _head_norm_bwd(s["k"], s["dk"], s["k_gain"], c, n)
    return (dq, dk) if dgq is None else (dq, dk, dgq, dgk)


def _tree(s):
    q, n_kv, hd = s["q"], s["k_cache"].shape[1], s["q"].shape[2]
    rep = q.shape[1] // n_kv
    past, cu = s["past"].long(), s["cu"].long()
    new, seqs, width, length = cu[1:] - cu[:-1], past.numel(), s["max_new"], s["max_kv"]
    node, key = torch.arange(width, device="cuda"), torch.arange(length, device="cuda")
    tok = (cu[:-1, None] + node).clamp(max=q.shape[0] - 1)                                        # [seqs, width]
    qp = q[tok].float().view(seqs, width, n_kv, rep, hd).permute(0, 2, 1, 3, 4).reshape(seqs, n_kv, width * rep, hd)
    held = key[None] < (past + new)[:, None]                                                      # [seqs, length]
    if s["table"] is not None:
        rows = s["table"].long()[:, key // PAGE] * PAGE + key % PAGE
    else:
        rows = s["row0"].long()[:, None] + key
    rows = torch.where(held, rows, torch.zeros_like(rows))

    def plane(cache, scale):
        x = (cache if scale is None else cache.view(torch.float8_e4m3fn))
        x = x.reshape(x.shape[0], -1).view(torch.uint8).view(x.shape[0], -1)[rows].view(x.dtype).float().view(seqs, length, n_kv, hd)
        return x if scale is None else x * scale[rows][:, :, None, None]

    scores = qp @ plane(s["k_cache"], s["k_scale"]).permute(0, 2, 3, 1) * (1.0 / math.sqrt(hd))
    at = key[None] - past[:, None]                                                                # key's place among the new tokens
    if s["mask"] is None:
        sees = at[:, None] <= node[None, :, None]
    else:
        words = s["mask"].shape[1]
        place = at.clamp(0, 32 * words - 1)
        word = s["mask"][tok].long().gather(2, (place // 32)[:, None].expand(-1, width, -1))
        sees = (at[:, None] < 0) | ((word >> (place % 32)[:, None]) & 1).bool()
    sees = (sees & held[:, None])[:, None, :, None].expand(-1, -1, -1, rep, -1).reshape(seqs, 1, width * rep, length)
    scores = torch.where(sees, scores, torch.full_like(scores, -math.inf))
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(scores - top)
    del scores
    total = p.sum(-1, keepdim=True)
    o = p @ plane(s["v_cache"], s["v_scale"]).permute(0, 2, 1, 3)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = top + torch.log(total)
    o = o.view(seqs, n_kv, width, rep, hd).permute(0, 2, 1, 3, 4).reshape(seqs, width, n_kv * rep, hd)
    lse = lse.view(seqs, n_kv, width, rep).permute(0, 2, 1, 3).reshape(seqs, width, n_kv * rep)
    b = torch.repeat_interleave(torch.arange(seqs, device="cuda"), new, output_size=q.shape[0])
    i = torch.arange(q.shape[0], device="cuda") - cu[b]
    return o[b, i].to(q.dtype), lse[b, i]


def _logprobs(s):
    case = s["case"]
    z = s["logits"].float() / case["temperature"]
    top = z.amax(1, keepdim=True)
    z -= top
    p = torch.exp(z)
    total = p.sum(1, keepdim=True)
    log_total = torch.log(total)
    # entropy: log(total) - sum p z / total with z relative to the row's largest; what has no probability adds nothing
    entropy = log_total[:, 0] - torch.where(p > 0, p * z, torch.zeros_like(z)).sum(1) / total[:, 0]
    del p
    targets = s["targets"].long()
    logprob = torch.where(targets >= 0, z.gather(1, targets.clamp(min=0)[:, None])[:, 0] - log_total[:, 0], torch.zeros_like(entropy))
    out = {"logprob": logprob, "entropy": entropy, "lse": (top + log_total)[:, 0]}
    if case["top"]:
        # the largest values; of equal ones the lowest index first: one whole number carries both
        bits = (s["logits"].float() + 0.0).view(torch.int32)
        keys = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + ((1 << 32) - 1 - torch.arange(z.shape[1], device="cuda"))
        ids = (1 << 32) - 1 - (keys.topk(case["top"], dim=1).values & ((1 << 32) - 1))
        out.update(top_ids=ids.to(torch.int32), top_logprobs=z.gather(1, ids) - log_total)
    return out


def _logprobs_bwd(s):
    t = s["case"]["temperature"]
    logp = s["logits"].float() / t - s["lse"][:, None]
    p = torch.exp(logp)
    d = -p * (s["g_logprob"] * (s["targets"] >= 0))[:, None] - torch.where(p > 0, p * (logp + s["entropy"][:, None]), torch.zeros_like(p)) * s["g_entropy"][:, None]
    hit = torch.where(s["targets"] >= 0, s["g_logprob"], torch.zeros_like(s["g_logprob"]))
    d.scatter_add_(1, s["targets"].long().clamp(min=0)[:, None], hit[:, None])
    return (d / t).to(s["logits"].dtype)


# ----------------------------------------------------------------------------------------------------------- passes
def _own(s):
    import paper_2410_03960_b200 as P
    op = s["op"]
    if op == "plan":
        P.plan_pages(s["past"], s["new"], s["owned"], s["table"], s["free"], s["n_free"], out=s["out"])
        return s["out"]
    if op == "rope":
        q = P.qk_norm_rope(s["q"], s["k"], s["v"], s["positions"], s["cos"], s["sin"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS, q_out=s["q_out"],
                           k_cache=s["k_cache"], v_cache=s["v_cache"], k_scale=s["k_scale"], v_scale=s["v_scale"], slot_map=s["slots"])
        if s["k_scale"] is None:
            return q, s["k_cache"], s["v_cache"]
        return q, s["k_cache"].view(torch.float8_e4m3fn), s["v_cache"].view(torch.float8_e4m3fn), s["k_scale"], s["v_scale"]
    if op == "rope_bwd":
        dq, dk, dgq, dgk = P.qk_norm_rope_bwd(s["dq"], s["dk"], s["q"], s["k"], s["positions"], s["cos"], s["sin"], q_gain=s["q_gain"], k_gain=s["k_gain"],
                                              eps=EPS, out=s["out"])
        return (dq, dk) if dgq is None else (dq, dk, dgq, dgk)
    if op == "tree":
        P.tree_attention(s["q"], s["k_cache"], s["v_cache"], s["past"], s["cu"], s["max_new"], s["max_kv"], block_table=s["table"], row0=s["row0"],
                         tree_mask=s["mask"], k_scale=s["k_scale"], v_scale=s["v_scale"], out=s["out"], lse=s["lse"])
        return s["out"], s["lse"]
    if op == "logprobs":
        P.token_logprobs(s["logits"], s["targets"], top_k=s["case"]["top"], temperature=s["case"]["temperature"], out=s["out"])
        return s["out"] if s["case"]["top"] else {k: s["out"][k] for k in ("logprob", "entropy", "lse")}
    return P.token_logprobs_bwd(s["logits"], s["targets"], s["lse"], s["entropy"], s["g_logprob"], s["g_entropy"], temperature=s["case"]["temperature"],
                                out=s["out"])


def run(state):
    if own:
        return _own(state)
    return {"plan": _plan, "rope": _rope, "rope_bwd": _rope_bwd, "tree": _tree, "logprobs": _logprobs, "logprobs_bwd": _logprobs_bwd}[state["op"]](state)


# ------------------------------------------------------------------------------------------------------ in 64 bits
def _spin(x, positions, hd, sign):
    """Pairs (i, i + hd/2) as complex numbers, turned by sign * position * theta^(-2 i / hd)."""
    angle = positions.double()[:, None] * THETA ** (-torch.arange(0, hd, 2, dtype=torch.float64, device="cuda") / hd)
    turned = torch.complex(x[..., : hd // 2], x[..., hd // 2:]) * torch.polar(torch.ones_like(angle), sign * angle)[:, None]
    return torch.cat([turned.real, turned.imag], -1)


def _exact_rope(s):
    hd = s["q"].shape[2]

    def head(x, gain):
        x = x.double()
        if gain is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / hd + EPS) * gain.double()
        return _spin(x, s["positions"], hd, 1.0)

    q, k, rows = head(s["q"], s["q_gain"]), head(s["k"], s["k_gain"]), s["slots"].long()
    if s["k_scale"] is None:
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
        kc[rows], vc[rows] = k, s["v"].double()
        return q, kc, vc
    ks, vs = s["k_scale"].double(), s["v_scale"].double()
    ks[rows], vs[rows] = k.flatten(1).abs().max(1).values / 448.0, s["v"].double().flatten(1).abs().max(1).values / 448.0
    return q, None, None, ks, vs                # the codes are whole steps: no value of their own in 64 bits


def _exact_rope_bwd(s):
    hd = s["q"].shape[2]

    def head(x, dy, gain):
        dz = _spin(dy.double(), s["positions"], hd, -1.0)
        if gain is None:
            return dz, None
        x = x.double()
        rms = torch.sqrt((x * x).sum(-1, keepdim=True) / hd + EPS)
        dn = dz * gain.double()
        return dn / rms - x * ((dn * x).sum(-1, keepdim=True) / hd) / rms ** 3, torch.einsum("thd,thd->d", dz, x / rms)

    dq, dgq = head(s["q"], s["dq"], s["q_gain"])
    dk, dgk = head(s["k"], s["dk"], s["k_gain"])
    return (dq, dk) if dgq is None else (dq, dk, dgq, dgk)


def _exact_tree(s):
    past, cu = s["past"].tolist(), s["cu"].tolist()
    n_kv, hd = s["k_cache"].shape[1], s["q"].shape[2]
    rep = s["q"].shape[1] // n_kv
    outs, lses = [], []
    for b, p in enumerate(past):
        n = cu[b + 1] - cu[b]
        if s["table"] is not None:
            rows = torch.cat([int(x) * PAGE + torch.arange(PAGE, device="cuda") for x in s["table"][b].tolist()[: -(-(p + n) // PAGE)]])[: p + n]
        else:
            rows = int(s["row0"][b]) + torch.arange(p + n, device="cuda")
        value = lambda c, sc: c[rows].double() if sc is None else c[rows].view(torch.float8_e4m3fn).double() * sc[rows].double()[:, None, None]  # noqa: E731
        k, v = value(s["k_cache"], s["k_scale"]), value(s["v_cache"], s["v_scale"])
        allowed = torch.ones((n, p + n), dtype=torch.bool, device="cuda")
        if s["mask"] is None:
            allowed[:, p:] = torch.tril(allowed[:, p:])
        else:
            bits = s["mask"][cu[b]: cu[b + 1]].long() & 0xFFFFFFFF
            allowed[:, p:] = torch.stack([(bits[:, i // 32] >> (i % 32)) & 1 for i in range(n)], 1).bool()
        o = torch.empty((n, n_kv * rep, hd), dtype=torch.float64, device="cuda")
        lse = torch.empty((n, n_kv * rep), dtype=torch.float64, device="cuda")
        for h in range(n_kv * rep):
            z = s["q"][cu[b]: cu[b + 1], h].double() @ k[:, h // rep].T / hd ** 0.5
            z = z.masked_fill(~allowed, -math.inf)
            lse[:, h] = torch.logsumexp(z, 1)
            o[:, h] = torch.softmax(z, 1) @ v[:, h // rep]
        outs.append(o)
        lses.append(lse)
    return torch.cat(outs), torch.cat(lses)


def _exact_logprobs(s):
    case, got = s["case"], {"logprob": [], "entropy": [], "lse": [], "top_logprobs": []}
    for r in range(0, case["rows"], 512):
        logp = torch.log_softmax(s["logits"][r: r + 512].double() / case["temperature"], 1)
        t = s["targets"][r: r + 512].long()
        got["logprob"].append(torch.where(t >= 0, logp.gather(1, t.clamp(min=0)[:, None])[:, 0], torch.zeros_like(logp[:, 0])))
        got["entropy"].append(-(logp.exp() * logp).sum(1))
        got["lse"].append((s["logits"][r: r + 512, 0].double() / case["temperature"]) - logp[:, 0])
        if case["top"]:
            got["top_logprobs"].append(logp.topk(case["top"], dim=1).values)
    out = {k: torch.cat(v) for k, v in got.items() if v}
    return {**out, "top_ids": None} if case["top"] else out


def _exact_logprobs_bwd(s):
    t, out = s["case"]["temperature"], []
    for r in range(0, s["case"]["rows"], 512):
        at = slice(r, r + 512)
        logp = s["logits"][at].double() / t - s["lse"][at].double()[:, None]
        p, hit = logp.exp(), s["targets"][at].long()
        known = (hit >= 0).double()
        one = torch.zeros_like(p).scatter_(1, hit.clamp(min=0)[:, None], known[:, None])
        d = s["g_logprob"][at].double()[:, None] * (one - p * known[:, None]) - s["g_entropy"][at].double()[:, None] * p * (logp + s["entropy"][at].double()[:, None])
        out.append(d / t)
    return torch.cat(out)


def exact(case, seed):
    if case["op"] == "plan":
        return None         # whole numbers: they have to be equal as they are
    s = prepare(case, seed)
    return {"rope": _exact_rope, "rope_bwd": _exact_rope_bwd, "tree": _exact_tree, "logprobs": _exact_logprobs, "logprobs_bwd": _exact_logprobs_bwd}[case["op"]](s)
