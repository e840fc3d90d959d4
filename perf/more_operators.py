"""Performance cases: attention to keys of another length, position biases, a shared prefix.

A decoder's queries attend to the states of an encoder, of another length and
padded to the longest of the batch (attn_cross_fwd, attn_cross_bwd: grouped
heads, views of fused projections, a length for each sequence). Models of that
kind learn a bias for each head and bucket of relative positions; the same calls
add it to the scores and return its gradient. A batch of sequences that begin
with the same long prompt keeps that prompt's keys and values once:
attn_prefix_decode appends a token to each sequence's own cache and attends to
the prefix and to it. Each is measured from the smallest call, where latency and
launches count, to the largest. Sizes are those of the workload tables in
``workloads`` and generic ones around them.

``run`` computes a case in its plain form, elementary torch operations in 32
bits (64 for the sums of a bias gradient), or through the library where ``own``
is true.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------- cases --
def _cross(name, train, B, Hq, Hkv, nq, nk, d, dtype, ragged, packed, causal=False, bias=None, empty=False):
    """`bias`: (buckets, distance from which on all share one, both directions) or None."""
    return {"name": name, "do": "train" if train else "forward", "B": B, "Hq": Hq, "Hkv": Hkv, "nq": nq, "nk": nk,
            "d": d, "dtype": dtype, "ragged": ragged, "empty": empty, "packed": packed, "causal": causal,
            "buckets": bias[0] if bias else 0, "distance": bias[1] if bias else 0, "both": bool(bias and bias[2])}


def _prefix(name, B, Hq, Hkv, np_, n, d, ragged):
    return {"name": name, "do": "prefix", "B": B, "Hq": Hq, "Hkv": Hkv, "np": np_, "n": n, "d": d, "ragged": ragged}


def listed():
    return [
        # a short description as the states, a small picture's positions as the queries: the smallest call
        _cross("cross_b1_h8_q64_k77_d64", False, 1, 8, 8, 64, 77, 64, "bf16", False, True),
        # the next token of a batch over the states of inputs of different lengths
        _cross("cross_b32_h16_q1_k1500_d64", False, 32, 16, 16, 1, 1500, 64, "bf16", True, False),
        # a training step: decoder texts against padded inputs, one projection for K and V
        _cross("cross_train_b8_h16_q448_k1500_d64", True, 8, 16, 16, 448, 1500, 64, "bf16", True, True),
        # a training step over long documents, grouped heads: the largest
        _cross("cross_train_b2_hq32_hkv8_q4096_k16384_d128", True, 2, 32, 8, 4096, 16384, 128, "bf16", False, False),
        # a float32 training step of a small model, odd lengths
        _cross("cross_train_b4_h8_q333_k1000_d64_f32", True, 4, 8, 8, 333, 1000, 64, "f32", True, False),
        # an encoder layer's training step, biased in both directions, padded inputs
        _cross("bias_train_b16_h8_n512_d64", True, 16, 8, 8, 512, 512, 64, "bf16", True, True, False, (32, 128, True)),
        # a decoder layer's training step, longer sequences, biased backwards only
        _cross("bias_train_b4_h16_n2048_d64_causal", True, 4, 16, 16, 2048, 2048, 64, "bf16", False, True, True,
               (32, 128, False)),
        # a float32 training step of a small biased model
        _cross("bias_train_b2_h8_n200_d32_f32", True, 2, 8, 8, 200, 200, 32, "f32", False, False, False, (32, 128, True)),
        # the next token of a batch of different lengths under the same bias
        _cross("bias_b16_h16_q1_k4096_d64", False, 16, 16, 16, 1, 4096, 64, "bf16", True, False, True, (32, 128, False)),
        # a few short chats behind one instruction
        _prefix("prefix_b4_hq8_hkv2_p1000_n100_d64", 4, 8, 2, 1000, 100, 64, False),
        # a large serving batch behind a long shared prompt, its own texts of different lengths
        _prefix("prefix_b64_hq64_hkv8_p8192_n512_d128", 64, 64, 8, 8192, 512, 128, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call of the listed ones' ranges."""
    do = rng.choice(["forward", "train", "train", "bias", "bias", "prefix"])
    while True:
        d = rng.choice([32, 64, 64, 128, 128])
        Hkv = rng.choice([1, 2, 4, 8, 8, 16])
        G = rng.choice([1, 1, 2, 4, 8])
        if do == "prefix":
            case = {"do": do, "B": _log_int(rng, 1, 64), "Hq": Hkv * G, "Hkv": Hkv, "np": _log_int(rng, 1, 16384),
                    "n": _log_int(rng, 1, 2048), "d": d, "ragged": rng.random() < 0.5}
            if case["B"] * case["n"] * Hkv * d <= 135_000_000 and case["B"] * Hkv * G * case["np"] <= 35_000_000:
                return case
            continue
        bias = do == "bias"
        train = do == "train" or (bias and rng.random() < 0.7)
        nk = _log_int(rng, 1, 8192 if bias else 16384)
        causal = bias and rng.random() < 0.5
        nq = nk if bias and train else 1 if rng.random() < 0.3 and not train else _log_int(rng, 1, 4096)
        if causal:
            nq = min(nq, nk)
        case = {"do": "train" if train else "forward", "B": _log_int(rng, 1, 32), "Hq": Hkv * G, "Hkv": Hkv, "nq": nq, "nk": nk,
                "d": d, "dtype": rng.choice(["bf16", "bf16", "f32"]), "ragged": rng.random() < 0.5,
                "empty": rng.random() < 0.15, "packed": rng.random() < 0.5, "causal": causal,
                "buckets": rng.choice([16, 32, 32, 64]) if bias else 0,
                "distance": rng.choice([64, 128, 128, 200]) if bias else 0, "both": bias and not causal}
        size = case["B"] * Hkv * G * nq * nk * d
        # the plain form holds the scores of a sequence, several times over
        if size <= (550_000_000_000 if case["dtype"] == "bf16" else 40_000_000_000) and Hkv * G * nq * nk <= 2_200_000_000:
            return case


# ------------------------------------------------------------------ inputs --
def _lengths(case, gen):
    """Lengths between a half and all of the longest, in some order; with `empty` one sequence has none."""
    B, n = case["B"], case["n" if case["do"] == "prefix" else "nk"]
    lens = [n - (n // 2) * i // B for i in range(B)] if case["ragged"] else [n] * B
    if case.get("empty"):
        lens[-1] = 0
    order = torch.randperm(B, generator=gen, device="cuda").tolist()
    return [lens[i] for i in order]


def _bucket_rows(buckets, distance, both):
    """The bucket of every relative position (key less query) between -distance and distance: half
    of a direction's buckets for the nearest positions, one each, the others at equal ratios up to
    `distance`; in whole numbers, so that a position on a border is where it belongs."""
    side = buckets // 2 if both else buckets
    near = side // 2
    far = side - near

    def bucket(p):
        if p < near:
            return p
        k = 0   # the largest with p >= near (distance / near)^(k / far)
        while k + 1 < far and p ** far >= near ** (far - k - 1) * distance ** (k + 1):
            k += 1
        return near + k
    return [bucket(-r) if r <= 0 else (side + bucket(r) if both else 0) for r in range(-distance, distance + 1)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    B, Hq, Hkv, d = case["B"], case["Hq"], case["Hkv"], case["d"]
    s = {"case": case, "scale": 1 / math.sqrt(d)}
    lens = _lengths(case, gen)
    if case["do"] == "prefix":
        qkv = normal(B, Hq + 2 * Hkv, d).to(torch.bfloat16)
        s["q"], s["k_new"], s["v_new"] = (x.contiguous() for x in (qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]))
        s["k_prefix"], s["v_prefix"] = (normal(Hkv, case["np"], d).to(torch.bfloat16) for _ in range(2))
        s["k_cache"], s["v_cache"] = (normal(B, Hkv, case["n"] + 1, d).to(torch.bfloat16) for _ in range(2))
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        return s
    dtype, nq, nk = DTYPES[case["dtype"]], case["nq"], case["nk"]
    q, kv = normal(B, nq, Hq, d).to(dtype).transpose(1, 2), normal(B, nk, 2 * Hkv, d).to(dtype).transpose(1, 2)
    s["q"], s["k"], s["v"] = q, kv[:, :Hkv], kv[:, Hkv:]   # as the projections give them
    if not case["packed"]:
        s["q"], s["k"], s["v"] = (s[x].contiguous() for x in ("q", "k", "v"))
    if case["do"] == "train":
        s["do"] = normal(B, Hq, nq, d).to(dtype)
    plain = case["ragged"] or case["empty"]
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda") if plain else None
    # the first query's position among the keys: a causal call's queries are a sequence's last tokens
    s["start"], s["starts"] = (nk - nq if case["causal"] else 0), None
    if case["causal"] and plain and nq < nk:
        s["start"], s["starts"] = 0, torch.tensor([x - nq for x in lens], dtype=torch.int32, device="cuda")
    if case["buckets"]:
        s["table"] = normal(case["buckets"], Hq).to(dtype)
        if own:
            import paper_2609_33916_amd as lib
            s["rows"], s["first"] = lib.attn_bias_buckets(case["buckets"], case["distance"], case["both"])
        else:
            rows = _bucket_rows(case["buckets"], case["distance"], case["both"])
            s["rows"], s["first"] = torch.tensor(rows, dtype=torch.int64, device="cuda"), -case["distance"]
    return s


# -------------------------------------------------------------- plain forms --
def _spread(x, G):
    """[Hkv, n, d] -> [Hkv * G, n, d] in 32 bits, a head for each query head."""
    return x.float().repeat_interleave(G, 0)


def _scores(s, b):
    """The scores [Hq, nq, nk] of one sequence, biased, -inf where a query does not see a key."""
    c = s["case"]
    x = s["q"][b].float() @ _spread(s["k"][b], c["Hq"] // c["Hkv"]).transpose(1, 2).contiguous()
    x *= s["scale"]
    start = s["start"] if s["starts"] is None else s["starts"][b]
    j = torch.arange(c["nk"], device="cuda")
    rel = j - (torch.arange(c["nq"], device="cuda") + start)[:, None]
    if c["buckets"]:
        rows = s["rows"][(rel - s["first"]).clamp(0, len(s["rows"]) - 1)]
        for h in range(c["Hq"]):
            x[h] += s["table"][:, h].float()[rows]
    seen = None
    if s["lens"] is not None:
        seen = (j < s["lens"][b]).expand(c["nq"], c["nk"])
    if c["causal"]:
        seen = rel <= 0 if seen is None else seen & (rel <= 0)
    if seen is not None:
        x.masked_fill_(~seen, -math.inf)
    return x


def _by_bucket(s, b, ds):
    """Sums [buckets, Hq] of ds [Hq, nq, nk] over the pairs of each bucket, in 64 bits: first over
    those of one relative position (a row one place further to the right than the next one's
    puts them below each other)."""
    c = s["case"]
    Hq, nq, nk = ds.shape
    wide = nq + nk - 1
    x = torch.zeros(Hq, nq, wide + 1, device="cuda")
    x[:, :, :nk] = ds.flip(1)
    x = x.flatten(1)[:, :nq * wide].unflatten(1, (nq, wide)).sum(1, dtype=torch.float64)
    start = s["start"] if s["starts"] is None else s["starts"][b]
    rel = torch.arange(wide, device="cuda") - (nq - 1) - start
    out = torch.zeros(c["buckets"], Hq, dtype=torch.float64, device="cuda")
    return out.index_add_(0, s["rows"][(rel - s["first"]).clamp(0, len(s["rows"]) - 1)], x.t().contiguous())


def _plain_cross(s):
    c = s["case"]
    B, Hq, Hkv, d, G = c["B"], c["Hq"], c["Hkv"], c["d"], c["Hq"] // c["Hkv"]
    dtype = s["q"].dtype
    o = torch.empty(B, Hq, c["nq"], d, dtype=dtype, device="cuda")
    lse = torch.empty(B, Hq, c["nq"], device="cuda")
    train = c["do"] == "train"
    if train:
        dq, dk, dv = (torch.empty(B, H, n, d, dtype=dtype, device="cuda")
                      for H, n in ((Hq, c["nq"]), (Hkv, c["nk"]), (Hkv, c["nk"])))
        dt = torch.zeros(c["buckets"], Hq, dtype=torch.float64, device="cuda")
    for b in range(B):
        p = _scores(s, b)
        top = p.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)   # finite where a row sees nothing
        p -= top
        p.exp_()
        z = p.sum(-1, keepdim=True)
        lse[b] = (top + z.log()).squeeze(-1)
        p /= z.clamp(min=torch.finfo(torch.float32).tiny)
        V = _spread(s["v"][b], G)
        out = p @ V
        o[b] = out.to(dtype)
        if not train:
            continue
        g = s["do"][b].float()
        pt = p.transpose(1, 2).contiguous()
        dv[b] = (pt @ g).unflatten(0, (Hkv, G)).sum(1).to(dtype)
        del pt
        ds = g @ V.transpose(1, 2).contiguous()
        ds -= (g * out).sum(-1, keepdim=True)
        ds *= p
        del p
        if c["buckets"]:
            dt += _by_bucket(s, b, ds)
        ds *= s["scale"]
        dq[b] = (ds @ _spread(s["k"][b], G)).to(dtype)
        ds = ds.transpose(1, 2).contiguous()
        dk[b] = (ds @ s["q"][b].float()).unflatten(0, (Hkv, G)).sum(1).to(dtype)
        del ds
    if not train:
        return o, lse
    return (o, lse, dq, dk, dv) + ((dt.to(dtype),) if c["buckets"] else ())


def _plain_prefix(s):
    c = s["case"]
    B, Hkv, G, d, at = c["B"], c["Hkv"], c["Hq"] // c["Hkv"], c["d"], s["lens"].long()
    b = torch.arange(B, device="cuda")
    s["k_cache"][b, :, at], s["v_cache"][b, :, at] = s["k_new"], s["v_new"]
    q = s["q"].float().unflatten(1, (Hkv, G)) * s["scale"]                         # [B, Hkv, G, d]
    qp = q.transpose(0, 1).flatten(1, 2)                                           # [Hkv, B G, d]
    xp = qp @ s["k_prefix"].float().transpose(1, 2).contiguous()                   # [Hkv, B G, np]
    xo = q @ s["k_cache"].float().transpose(2, 3).contiguous()                     # [B, Hkv, G, n + 1]
    seen = torch.arange(c["n"] + 1, device="cuda") <= s["lens"][:, None, None, None]
    xo = torch.where(seen, xo, -math.inf)
    top = torch.maximum(xp.amax(-1).unflatten(1, (B, G)).transpose(0, 1), xo.amax(-1))[..., None]   # [B, Hkv, G, 1]
    pp = (xp - top.transpose(0, 1).flatten(1, 2)).exp()
    po = (xo - top).exp()
    z = pp.sum(-1).unflatten(1, (B, G)).transpose(0, 1)[..., None] + po.sum(-1, keepdim=True)
    o = (pp @ s["v_prefix"].float()).unflatten(1, (B, G)).transpose(0, 1) + po @ s["v_cache"].float()
    return (o / z).flatten(1, 2).to(torch.bfloat16), (top + z.log()).flatten(1), s["k_cache"], s["v_cache"]


# --------------------------------------------------------------------- run --
def run(s):
    if s["case"]["do"] == "prefix":
        return _own_prefix(s) if own else _plain_prefix(s)
    return _own_cross(s) if own else _plain_cross(s)


def _own_cross(s):
    import paper_2609_33916_amd as lib
    c = s["case"]
    how = {"scale": s["scale"], "causal": c["causal"], "start": s["start"], "starts": s["starts"], "k_lens": s["lens"]}
    if c["buckets"]:
        how.update(bias=s["table"], bias_rows=s["rows"], bias_first=s["first"])
    o, lse = lib.attn_cross_fwd(s["q"], s["k"], s["v"], **how)
    if c["do"] != "train":
        return o, lse
    return (o, lse) + tuple(lib.attn_cross_bwd(s["q"], s["k"], s["v"], o, lse, s["do"], **how))


def _own_prefix(s):
    import paper_2609_33916_amd as lib
    o, lse = lib.attn_prefix_decode(s["q"], s["k_prefix"], s["v_prefix"], s["k_cache"], s["v_cache"], k_new=s["k_new"],
                                    v_new=s["v_new"], cache_lens=s["lens"], n=s["case"]["n"], scale=s["scale"])
    return o, lse, s["k_cache"], s["v_cache"]


# -------------------------------------------------------------------- work --
def work(case):
    B, Hq, Hkv, d = case["B"], case["Hq"], case["Hkv"], case["d"]
    n = case["n"] if case["do"] == "prefix" else case["nk"]
    lens = [n - (n // 2) * i // B for i in range(B)] if case["ragged"] else [n] * B
    if case.get("empty"):
        lens[-1] = 0
    if case["do"] == "prefix":
        own_rows = sum(lens) + B
        return {"bytes": 4 * Hkv * d * (case["np"] + own_rows + B) + 4 * B * Hq * d + 4 * B * Hq,
                "flops": 4 * Hq * d * (B * case["np"] + own_rows)}
    nq, nk = case["nq"], case["nk"]
    e = 2 if case["dtype"] == "bf16" else 4
    pairs = 0   # of a query and a key that it sees, for one head
    for x in lens:
        if not case["causal"]:
            pairs += nq * x
            continue
        first = (x if nq < nk else nk) - nq   # the first query's position; it sees keys up to there
        full = max(0, min(nq, first + nq - x))   # queries behind the last key see all of them
        part = nq - full
        pairs += full * x + sum(max(0, first + i + 1) for i in range(part))
    train = case["do"] == "train"
    rows_q, rows_k = B * Hq * nq * d, Hkv * d * sum(lens)
    moved = e * (2 * rows_q + 2 * rows_k) + 4 * B * Hq * nq
    if train:   # and dO, dQ; dK and dV with the zeros of the padding
        moved += e * (2 * rows_q + 2 * B * Hkv * nk * d)
    moved += (2 if train else 1) * e * case["buckets"] * Hq
    return {"bytes": moved, "flops": (14 if train else 4) * Hq * d * pairs}


# ------------------------------------------------------------------- exact --
def _exact_bucket(rel, buckets, distance, both):
    """The bucket of relative positions (whole numbers, any shape), from logarithms in 64 bits; a
    logarithm within 1e-9 below a border counts as on it."""
    side = buckets // 2 if both else buckets
    near = side // 2
    back = torch.clamp(-rel, min=0) if not both else rel.abs()
    t = torch.log(back.clamp(min=1).double() / near) / math.log(distance / near) * (side - near)
    far = near + torch.floor(t + 1e-9).long().clamp(max=side - near - 1)
    out = torch.where(back < near, back, far)
    return out + side * (rel > 0).long() if both else out


def _exact_cross(case, s):
    B, Hq, G, nq, nk, d = case["B"], case["Hq"], case["Hq"] // case["Hkv"], case["nq"], case["nk"], case["d"]
    train = case["do"] == "train"
    f = {"dtype": torch.float64, "device": "cuda"}
    o, lse = torch.zeros(B, Hq, nq, d, **f), torch.full((B, Hq, nq), -math.inf, **f)
    dq, dk, dv = torch.zeros(B, Hq, nq, d, **f), torch.zeros(B, case["Hkv"], nk, d, **f), torch.zeros(B, case["Hkv"], nk, d, **f)
    dt = torch.zeros(case["buckets"], Hq, **f)
    step = max(1, 100_000_000 // nk)   # queries at once
    for b in range(B):
        n = nk if s["lens"] is None else int(s["lens"][b])
        start = int(s["start"] if s["starts"] is None else s["starts"][b])
        if n == 0:
            continue
        for h in range(Hq):
            K, V = s["k"][b, h // G, :n].double(), s["v"][b, h // G, :n].double()
            for i0 in range(0, nq, step):
                Q = s["q"][b, h, i0:i0 + step].double()
                rel = torch.arange(n, device="cuda")[None] - torch.arange(start + i0, start + i0 + len(Q), device="cuda")[:, None]
                w = torch.mm(Q, K.t().contiguous()).mul_(s["scale"])
                if case["buckets"]:
                    bucket = _exact_bucket(rel, case["buckets"], case["distance"], case["both"])
                    w += s["table"][:, h].double()[bucket]
                if case["causal"]:
                    w[rel > 0] = -math.inf
                L = torch.logsumexp(w, 1, keepdim=True)
                lse[b, h, i0:i0 + step] = L[:, 0]
                w = torch.where(L == -math.inf, torch.zeros_like(w), torch.exp(w - L))
                y = torch.mm(w, V)
                o[b, h, i0:i0 + step] = y
                if not train:
                    continue
                dO = s["do"][b, h, i0:i0 + step].double()
                dv[b, h // G, :n] += torch.mm(w.t().contiguous(), dO)
                w *= torch.mm(dO, V.t().contiguous()) - (dO * y).sum(1, keepdim=True)
                if case["buckets"]:
                    dt[:, h] += torch.bincount(bucket.flatten(), w.flatten(), minlength=case["buckets"])
                dq[b, h, i0:i0 + step] = s["scale"] * torch.mm(w, K)
                dk[b, h // G, :n] += s["scale"] * torch.mm(w.t().contiguous(), Q)
    if not train:
        return o, lse
    return (o, lse, dq, dk, dv) + ((dt,) if case["buckets"] else ())


def exact(case, seed):
    s = prepare(case, seed)
    if case["do"] != "prefix":
        return _exact_cross(case, s)
    B, Hq, Hkv, d = case["B"], case["Hq"], case["Hkv"], case["d"]
    o = torch.empty(B, Hq, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(B, Hq, dtype=torch.float64, device="cuda")
    caches = [s["k_cache"].double(), s["v_cache"].double()]
    for b, n in enumerate(s["lens"].tolist()):
        for x, new in zip(caches, (s["k_new"], s["v_new"])):
            x[b, :, n] = new[b].double()
        K, V = (torch.cat((s[p].double(), x[b, :, :n + 1]), 1) for p, x in zip(("k_prefix", "v_prefix"), caches))
        w = torch.bmm(s["q"][b].double().reshape(Hkv, -1, d), K.transpose(1, 2).contiguous()) * s["scale"]
        lse[b] = torch.logsumexp(w, 2).flatten()
        o[b] = torch.bmm(torch.softmax(w, 2), V).reshape(Hq, d)
    return o, lse, *caches
