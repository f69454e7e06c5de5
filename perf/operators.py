"""The operators of one decode layer, as they are measured: their inputs, their plain forms and their exact values.

Four operators that a serving plan prices per layer and step: the residual addition with its root-mean-square norm and
an 8-bit output ("norm"), the writing of new keys and values into an 8-bit paged cache ("append"), single-token
attention over that cache ("attention") and a whole mixture-of-experts layer for a few tokens ("moe").

`run` computes them with elementary torch operations in 32 bits where `own` is false, and through the framework's
public calls where it is true.  The 8-bit tensors are torch.float8_e4m3fn, so what comes back are the values the bytes
stand for.  Sequence lengths follow from the case alone (a low-discrepancy sequence), everything else from the seed.
"""
import math

import torch

own = False

DEV = "cuda"
F8 = torch.float8_e4m3fn
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4, "e4m3": 1}
F8_MAX = 448.0
EPS = 1e-6
BLOCK = 128          # side of a weight-scale block, and of an activation-scale group


def listed():
    return [
        # one token through the widest of the modeled stacks: nothing but latency
        dict(name="norm 1x7168", op="norm", rows=1, hidden=7168, dtype="bf16", group=128, residual=True),
        # an odd decode batch, one scale a row, half precision
        dict(name="norm 509x5120 row", op="norm", rows=509, hidden=5120, dtype="f16", group=0, residual=True),
        # a prompt chunk: bandwidth
        dict(name="norm 8192x7168", op="norm", rows=8192, hidden=7168, dtype="bf16", group=128, residual=True),
        # a decode step's new token of each of many sequences
        dict(name="append 256x1", op="append", seqs=256, new_lo=1, new_hi=1, past_hi=511, kv_heads=32, head_dim=128, page=64),
        # prompts of several requests, ragged, some behind an already cached prefix
        dict(name="append 6 prompts", op="append", seqs=6, new_lo=17, new_hi=4096, past_hi=300, kv_heads=8, head_dim=128, page=64),
        # a single short request on the smallest model: latency
        dict(name="attention 1x777", op="attention", seqs=1, len_lo=777, len_hi=777, heads=16, kv_heads=16, head_dim=64, page=16),
        # an ordinary ragged decode batch with shared heads
        dict(name="attention 48x8k", op="attention", seqs=48, len_lo=1, len_hi=8192, heads=32, kv_heads=8, head_dim=128, page=64),
        # one very long context: the split over the length
        dict(name="attention 1x131k", op="attention", seqs=1, len_lo=131071, len_hi=131071, heads=64, kv_heads=8, head_dim=128, page=64),
        # single-token decode, all experts on this GPU
        dict(name="moe bf16 1", op="moe", tokens=1, hidden=4096, ffn=1408, experts=64, local=64, first=0, top_k=6, shared=2, weights="bf16"),
        # a few tokens on few experts: several tokens an expert
        dict(name="moe bf16 29", op="moe", tokens=29, hidden=1024, ffn=2816, experts=8, local=8, first=0, top_k=2, shared=0, weights="bf16"),
        # a quarter of the experts on this GPU, 8-bit weights
        dict(name="moe e4m3 16", op="moe", tokens=16, hidden=5120, ffn=1536, experts=128, local=32, first=32, top_k=8, shared=1, weights="e4m3"),
        # an eighth of the experts of the largest stack, a decode batch
        dict(name="moe e4m3 128", op="moe", tokens=128, hidden=7168, ffn=2048, experts=256, local=32, first=96, top_k=8, shared=1, weights="e4m3"),
    ]


def log_int(rng, lo, hi):
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return n - (n == 3 << 10)


def draw(rng):
    op = rng.choice(["norm", "append", "attention", "attention", "moe", "moe"])
    if op == "norm":
        return dict(op=op, rows=log_int(rng, 1, 8192), hidden=rng.choice([1024, 4096, 5120, 7168, 8 * (2 * log_int(rng, 8, 447) + 1), 2 * log_int(rng, 8, 3583) + 1]), dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    group=rng.choice([0, 128]), residual=rng.random() < 0.8)   # odd widths too: rows that start unaligned
    if op == "append":
        new = log_int(rng, 1, 2048)
        return dict(op=op, seqs=log_int(rng, 1, max(1, min(256, 8192 // new))), new_lo=rng.choice([0, 1, new]), new_hi=new, past_hi=rng.choice([0, 63, 511]),
                    kv_heads=rng.choice([1, 2, 4, 8, 16]), head_dim=rng.choice([64, 128]), page=rng.choice([16, 32, 64, 128]))
    if op == "attention":
        kv_heads, head_dim = rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([64, 128])
        top = log_int(rng, 1, 65536)
        most = max(1, min(256, (1 << 28) // (top * kv_heads * head_dim * 2)))
        return dict(op=op, seqs=log_int(rng, 1, most), len_lo=rng.choice([0, 1, top]), len_hi=top, heads=kv_heads * rng.choice([1, 2, 4, 5, 8, 16]), kv_heads=kv_heads,
                    head_dim=head_dim, page=rng.choice([16, 32, 64, 128]))
    hidden, ffn, experts, top_k, shared = rng.choice([(1024, 2816, 8, 2, 0), (4096, 1408, 64, 6, 2), (5120, 1536, 128, 8, 1), (7168, 2048, 256, 8, 1)])
    parts = rng.choice([p for p in (1, 2, 4, 8) if 2 <= experts // p <= 64])
    local = experts // parts
    if rng.random() < 0.4:
        ffn = 8 * log_int(rng, 11, ffn // 8) + rng.choice([0, 0, 3])      # a slice of the experts' width, odd ones too
    return dict(op=op, tokens=log_int(rng, 1, 128 if hidden > 4096 or experts > 64 else 64), hidden=hidden, ffn=ffn, experts=experts, local=local,
                first=local * rng.randrange(parts), top_k=top_k, shared=shared, weights=rng.choice(["bf16", "e4m3"]) if local <= 32 else "e4m3")


# ------------------------------------------------------------------ shapes that follow from a case
def spread(n, lo, hi, shift=0.0):
    """n whole numbers in [lo, hi], evenly but irregularly spread, the first at the upper end."""
    return [hi - int(((i * 0.6180339887498949 + shift) % 1.0) * (hi - lo + 1)) if hi > lo else hi for i in range(n)]


def append_shape(c):
    new = spread(c["seqs"], c["new_lo"], c["new_hi"])
    past = spread(c["seqs"], 0, c["past_hi"], 0.25)
    cols = max(-(-(p + n) // c["page"]) for p, n in zip(past, new)) + 1
    return new, past, cols


def attention_shape(c):
    lens = spread(c["seqs"], c["len_lo"], c["len_hi"])
    return lens, max(1, -(-max(lens) // c["page"]))


def experts_touched(c):
    """Expected number of local experts that at least one token chose."""
    return c["local"] * (1.0 - (1.0 - c["top_k"] / c["experts"]) ** c["tokens"]) + c["shared"]


def work(case):
    c = case
    if c["op"] == "norm":
        n, b = c["rows"] * c["hidden"], BYTES[c["dtype"]]
        groups = c["rows"] * (1 if c["group"] == 0 else -(-c["hidden"] // c["group"]))
        # x and the residual in; the sum, the norm and its 8-bit form out
        return {"bytes": n * b * (2 + 2 * c["residual"]) + n + 4 * groups + c["hidden"] * b, "flops": 8 * n}
    if c["op"] == "append":
        n = sum(append_shape(c)[0]) * c["kv_heads"] * c["head_dim"] * 2
        return {"bytes": 3 * n, "flops": 4 * n}
    if c["op"] == "attention":
        lens, _ = attention_shape(c)
        tok, d = sum(lens), c["head_dim"]
        scales = sum(-(-n // c["page"]) for n in lens) * c["kv_heads"] * 8
        return {"bytes": tok * c["kv_heads"] * d * 2 + scales + 4 * c["seqs"] * c["heads"] * d, "flops": 4 * tok * c["heads"] * d}
    pairs = c["tokens"] * (c["top_k"] * c["local"] / c["experts"] + c["shared"])
    mat = 3 * c["ffn"] * c["hidden"]
    return {"bytes": experts_touched(c) * mat * BYTES[c["weights"]] + c["experts"] * c["hidden"] * 2 + c["tokens"] * c["hidden"] * 4,
            "flops": 2 * pairs * mat + 2 * c["tokens"] * c["experts"] * c["hidden"]}


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device=DEV) * std).to(dtype)

    def bytes8(*shape):
        # 8-bit values as a scaled normal tensor has them: the largest of a block near the end of the range
        return normal(*shape, std=120.0).clamp_(-F8_MAX, F8_MAX).to(F8)

    s = dict(c)
    if c["op"] == "norm":
        dt = DTYPES[c["dtype"]]
        s["x"] = normal(c["rows"], c["hidden"], dtype=dt)
        s["residual"] = normal(c["rows"], c["hidden"], std=3.0, dtype=dt) if c["residual"] else None
        s["weight"] = (1.0 + normal(c["hidden"], std=0.2)).to(dt)
    elif c["op"] in ("append", "attention"):
        if c["op"] == "append":
            new, past, cols = append_shape(c)
            lens = past
            s["cu_new"] = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32, device=DEV)
            s["max_new"] = max(new)
            s["k"], s["v"] = (normal(sum(new), c["kv_heads"], c["head_dim"], std=w, dtype=torch.bfloat16) for w in (2.0, 0.7))
        else:
            lens, cols = attention_shape(c)
            s["query"] = normal(c["seqs"], c["heads"], c["head_dim"], dtype=torch.bfloat16)
            s["sm_scale"] = 1.0 / math.sqrt(c["head_dim"])
        n_pages = c["seqs"] * cols + 3
        shape = (n_pages, c["kv_heads"], c["page"], c["head_dim"])
        s["table"] = torch.randperm(n_pages, generator=g, device=DEV)[:c["seqs"] * cols].reshape(c["seqs"], cols).to(torch.int32)
        s["lengths"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        s["k_cache"], s["v_cache"] = bytes8(*shape), bytes8(*shape)
        # powers of two, as the append writes them
        s["k_scale"], s["v_scale"] = (torch.exp2(torch.randint(lo, lo + 3, shape[:2], generator=g, device=DEV).float()) for lo in (-8, -9))
    else:
        H, F, E, n = c["hidden"], c["ffn"], c["experts"], c["local"] + c["shared"]
        s["x"] = normal(c["tokens"], H, dtype=torch.bfloat16)
        s["router"] = normal(E, H, std=1.0 / math.sqrt(H), dtype=torch.bfloat16)
        names, shapes = ("gate", "up", "down"), ((n, F, H), (n, F, H), (n, H, F))
        if c["weights"] == "bf16":
            for name, shape in zip(names, shapes):
                s[name] = normal(*shape, std=1.0 / math.sqrt(shape[2]), dtype=torch.bfloat16)
                s[name + "_scale"] = None
            s["xq"] = s["xq_scale"] = None
        else:
            for name, shape in zip(names, shapes):
                s[name] = bytes8(*shape)
                blocks = (n, -(-shape[1] // BLOCK), -(-shape[2] // BLOCK))
                s[name + "_scale"] = torch.exp2(torch.rand(*blocks, generator=g, device=DEV) - 0.5) / (120.0 * math.sqrt(shape[2]))
            # the tokens in 8 bits as the norm in front of the layer writes them
            groups = s["x"].float().reshape(c["tokens"], -1, BLOCK)
            scale = groups.abs().amax(-1) / F8_MAX
            s["xq"], s["xq_scale"] = (groups / scale[..., None]).reshape(c["tokens"], H).to(F8), scale
        if own:   # a program that serves lays its weights out once, and keeps them so
            from paper_2607_18631_b200 import ops
            s["layer"] = ops.MoeLayer(s["router"], s["gate"], s["up"], s["down"], top_k=c["top_k"], first_expert=c["first"], n_shared=c["shared"],
                                      gate_scale=s["gate_scale"], up_scale=s["up_scale"], down_scale=s["down_scale"])
    return s


# ------------------------------------------------------------------ one pass
def run(state):
    s = state
    if own:
        from paper_2607_18631_b200 import ops
        if s["op"] == "norm":
            return ops.pf_add_rms_norm(s["x"], s["residual"], s["weight"], eps=EPS, group=s["group"], y=True)
        if s["op"] == "append":
            ops.pf_kv_append(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["k"], s["v"], s["cu_new"], s["lengths"], s["table"], max_new=s["max_new"])
            return {n: s[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale")}
        if s["op"] == "attention":
            return ops.pf_decode_attention(s["query"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["lengths"], s["table"], sm_scale=s["sm_scale"], lse=True)
        return s["layer"].forward(s["x"], s["xq"], s["xq_scale"])
    return {"norm": plain_norm, "append": plain_append, "attention": plain_attention, "moe": plain_moe}[s["op"]](s)


def plain_norm(s):
    dt = s["x"].dtype
    a = s["x"].float() if s["residual"] is None else s["x"].float() + s["residual"].float()
    y = a * torch.rsqrt(a.square().mean(-1, keepdim=True) + EPS) * s["weight"].float()
    T, H = y.shape
    width = s["group"] or H
    n = -(-H // width)
    padded = torch.zeros(T, n * width, device=DEV)
    padded[:, :H] = y
    amax = padded.reshape(T, n, width).abs().amax(-1)
    scale = torch.where(amax > 0, (amax / F8_MAX).clamp(min=2.0 ** -100), torch.ones_like(amax))
    q = (padded.reshape(T, n, width) / scale[..., None]).clamp(-F8_MAX, F8_MAX).reshape(T, n * width)[:, :H].to(F8)
    out = {"y": y.to(dt), "q": q, "scale": scale}
    if s["residual"] is not None:
        out["sum"] = a.to(dt)
    return out


def pow2_scale(amax):
    """The least power of two that brings amax into the 8-bit range, 2^-100 at least."""
    m, e = torch.frexp(amax)
    e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.ldexp(torch.ones_like(amax), torch.where(amax > 0, e, -100).clamp(-100, 118))


def plain_append(s):
    P = s["page"]
    cu, lens, table = s["cu_new"].long(), s["lengths"].long(), s["table"].long()
    n_new = cu[1:] - cu[:-1]
    seq = torch.repeat_interleave(torch.arange(s["seqs"], device=DEV), n_new, output_size=s["k"].shape[0])
    pos = lens[seq] + torch.arange(s["k"].shape[0], device=DEV) - cu[seq]
    page, slot = table[seq, pos // P], pos % P
    # the only page of a sequence that can hold earlier tokens is the one its first new token falls into
    head = table.gather(1, (lens // P).clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    before = torch.where(n_new > 0, lens % P, 0)
    kept = (torch.arange(P, device=DEV)[None, :] < before[:, None])[:, None, :, None]
    for cache, scale, x in ((s["k_cache"], s["k_scale"], s["k"].float()), (s["v_cache"], s["v_scale"], s["v"].float())):
        raw = cache.view(torch.uint8)
        amax = torch.zeros_like(scale).index_reduce_(0, page, x.abs().amax(-1), "amax")
        touched = torch.zeros(scale.shape[0], dtype=torch.bool, device=DEV).index_fill_(0, page, True)
        new_scale = torch.where(touched[:, None], pow2_scale(amax), scale)
        old = scale[head]
        joint = torch.where((before > 0)[:, None], torch.maximum(old, new_scale[head]), new_scale[head])
        new_scale[head] = joint
        values = cache[head].float() * (old / joint)[:, :, None, None]
        raw[head] = torch.where(kept, values.to(F8).view(torch.uint8), raw[head])
        raw[page, :, slot] = (x / new_scale[page][..., None]).clamp(-F8_MAX, F8_MAX).to(F8).view(torch.uint8)
        scale.copy_(new_scale)
    return {n: s[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale")}


def plain_attention(s):
    B, nh, d = s["query"].shape
    nkv, P, cols = s["kv_heads"], s["page"], s["table"].shape[1]
    at = s["table"].long()

    def dense(cache, scale):
        x = cache.view(torch.uint8)[at].view(F8).float() * scale[at][..., None, None]      # [B, cols, nkv, P, d]
        return x.permute(0, 2, 1, 3, 4).reshape(B, nkv, cols * P, d)

    q = s["query"].float().reshape(B, nkv, nh // nkv, d)
    score = torch.matmul(q, dense(s["k_cache"], s["k_scale"]).transpose(2, 3)) * s["sm_scale"]
    seen = torch.arange(cols * P, device=DEV)[None, :] < s["lengths"].long()[:, None]
    score = score.masked_fill(~seen[:, None, None, :], float("-inf"))
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), 0.0, top)
    e = torch.exp(score - top)
    total = e.sum(-1, keepdim=True)
    out = torch.matmul(e, dense(s["v_cache"], s["v_scale"])) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total)).reshape(B, nh)
    return {"out": out.reshape(B, nh, d).to(s["query"].dtype), "lse": lse}


def spread_scale(scale, rows, cols):
    return scale.repeat_interleave(BLOCK, 1)[:, :rows].repeat_interleave(BLOCK, 2)[:, :, :cols]


def plain_moe(s):
    T, K, local, shared = s["tokens"], s["top_k"], s["local"], s["shared"]
    logits = torch.matmul(s["x"].float(), s["router"].float().t())
    top, ids = torch.sort(logits, dim=-1, descending=True, stable=True)
    top, ids = top[:, :K], ids[:, :K]
    share = torch.exp(top - top[:, :1])
    share = share / share.sum(-1, keepdim=True)
    mix = torch.zeros(T, s["experts"], device=DEV).scatter_(1, ids, share)[:, s["first"]:s["first"] + local]
    mix = torch.cat([mix, torch.ones(T, shared, device=DEV)], 1)                              # [T, local + shared]
    if s["xq"] is None:
        x, (gate, up, down) = s["x"].float(), (s[n].float() for n in ("gate", "up", "down"))
    else:
        x = s["xq"].float() * s["xq_scale"].repeat_interleave(BLOCK, 1)[:, :s["hidden"]]
        gate, up, down = (s[n].float() * spread_scale(s[n + "_scale"], s[n].shape[1], s[n].shape[2]) for n in ("gate", "up", "down"))
    g, u = torch.matmul(x, gate.transpose(1, 2)), torch.matmul(x, up.transpose(1, 2))         # [experts, T, ffn]
    h = g / (1.0 + torch.exp(-g)) * u * mix.t()[:, :, None]
    out = torch.matmul(h, down.transpose(1, 2)).sum(0)
    return {"out": out.to(torch.bfloat16), "ids": ids.to(torch.int32), "weights": share}


# ------------------------------------------------------------------ 64-bit values
def exact(case, seed):
    """What `run` returns, from the definitions in 64 bits; 8-bit outputs before their rounding, whole numbers left out."""
    c = case
    s = {k: v for k, v in prepare(c, seed).items() if k != "layer"}
    f64 = torch.float64
    if c["op"] == "norm":
        a = s["x"].to(f64)
        if c["residual"]:
            a = a + s["residual"].to(f64)
        y = a / (a.pow(2).sum(-1) / c["hidden"] + EPS).sqrt().unsqueeze(-1) * s["weight"].to(f64)
        step = c["group"] or c["hidden"]
        parts = torch.split(y, step, dim=1)
        scale = torch.stack([p.abs().max(1).values / F8_MAX for p in parts], 1)
        q = torch.cat([p / scale[:, i:i + 1] for i, p in enumerate(parts)], 1)
        out = {"y": y, "q": q, "scale": scale}
        return {**out, "sum": a} if c["residual"] else out
    if c["op"] == "append":
        new, past, _ = append_shape(c)
        table, P, at, out = s["table"].tolist(), c["page"], 0, {}
        rows = []          # (page, first slot, last slot, first token of k / v)
        for b, (n, p) in enumerate(zip(new, past)):
            j = 0
            while j < n:
                slot = (p + j) % P
                m = min(P - slot, n - j)
                rows.append((table[b][(p + j) // P], slot, slot + m, at + j))
                j += m
            at += n
        for name, x in (("k", s["k"]), ("v", s["v"])):
            values, scale = s[name + "_cache"].to(f64), s[name + "_scale"].to(f64)
            for page, lo, hi, t in rows:
                part = x[t:t + hi - lo].to(f64).transpose(0, 1)                               # [heads, tokens, head_dim]
                need = torch.exp2(torch.ceil(torch.log2(part.abs().amax((1, 2)) / F8_MAX) - 1e-9))   # 7.0 / 448 is a power of two
                now = torch.maximum(need, scale[page]) if lo else need
                values[page, :, :lo] *= (scale[page] / now)[:, None, None]
                values[page, :, lo:hi] = part / now[:, None, None]
                scale[page] = now
            out[name + "_cache"], out[name + "_scale"] = values, scale
        return out
    if c["op"] == "attention":
        lens, _ = attention_shape(c)
        G, d = c["heads"] // c["kv_heads"], c["head_dim"]
        out = torch.zeros(c["seqs"], c["heads"], d, dtype=f64, device=DEV)
        lse = torch.full((c["seqs"], c["heads"]), float("-inf"), dtype=f64, device=DEV)
        for b, n in enumerate(lens):
            if n == 0:
                continue
            pages = s["table"][b, :-(-n // c["page"])].long()
            for h in range(c["kv_heads"]):
                k, v = ((s[m + "_cache"][:, h].view(torch.uint8)[pages].view(F8).to(f64) * s[m + "_scale"][pages, h].to(f64)[:, None, None]).reshape(-1, d)[:n] for m in ("k", "v"))
                score = s["query"][b, h * G:(h + 1) * G].to(f64) @ k.T * s["sm_scale"]
                lse[b, h * G:(h + 1) * G] = torch.logsumexp(score, -1)
                out[b, h * G:(h + 1) * G] = torch.softmax(score, -1) @ v
        return {"out": out, "lse": lse}
    T, local = c["tokens"], c["local"]
    logits = s["x"].to(f64) @ s["router"].to(f64).T
    chosen = torch.sort(logits, dim=-1, descending=True, stable=True)
    ids, share = chosen.indices[:, :c["top_k"]], torch.softmax(chosen.values[:, :c["top_k"]], -1)
    x = s["x"].to(f64) if s["xq"] is None else (s["xq"].to(f64).reshape(T, -1, BLOCK) * s["xq_scale"].to(f64).unsqueeze(-1)).reshape(T, -1)

    def matrix(name, e):
        w = s[name][e].to(f64)
        if s["xq"] is not None:
            rows, cols = (torch.arange(n, device=DEV) // BLOCK for n in w.shape)
            w = w * s[name + "_scale"][e].to(f64)[rows][:, cols]
        return w

    out = torch.zeros(T, c["hidden"], dtype=f64, device=DEV)
    for e in range(local + c["shared"]):
        part = (share * (ids == c["first"] + e)).sum(1) if e < local else torch.ones(T, dtype=f64, device=DEV)
        rows = part.nonzero()[:, 0]
        if rows.numel():
            g = x[rows] @ matrix("gate", e).T
            h = g * torch.sigmoid(g) * (x[rows] @ matrix("up", e).T)
            out[rows] += part[rows, None] * (h @ matrix("down", e).T)
    return {"out": out, "ids": None, "weights": share}
