"""Rotary positions, the cache append that applies them, and attention over a shared prefix, as they are measured: inputs, plain forms and exact values.

Three operators around the 8-bit paged cache: the rotation of query and key heads by their positions and its gradient ("rope"), the
writing of new keys and values into the cache with the rotation on the way ("append"), and single-token attention of
sequences that share long prefixes ("prefix").

`run` computes them with elementary torch operations in 32 bits (angles in 64) where `own` is false, and through the framework's public calls where
it is true.  The 8-bit tensors are torch.float8_e4m3fn, so what comes back are the values the bytes stand for.  Lengths follow from the
case alone (a low-discrepancy sequence), everything else from the seed.
"""
import math

import torch

own = False

DEV = "cuda"
F8 = torch.float8_e4m3fn
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
F8_MAX = 448.0
MOST = 1 << 29       # rows times prefix tokens of a drawn case: no more than the largest listed one has


def listed():
    plain = dict(layout="half", base=10000.0, scaling="none", factor=1.0, original=8192, amplitude=1.0)
    long = dict(layout="half", base=500000.0, scaling="parts", factor=8.0, original=8192, amplitude=1.0)
    return [
        # one decode token's query heads: nothing but latency
        dict(name="rope 1x32x128", op="rope", tokens=1, heads=32, head_dim=128, rot=128, dtype="bf16", far=8191, transposed=False, **plain),
        # a ragged prompt chunk, an odd number of heads, a quarter of each rotated, neighbouring pairs
        dict(name="rope 4099x25x64 quarter", op="rope", tokens=4099, heads=25, head_dim=64, rot=16, dtype="f16", far=32767, transposed=False, **{**plain, "layout": "interleaved"}),
        # the gradient of a training batch, far positions of a long context
        dict(name="rope 8192x40x128 gradient", op="rope", tokens=8192, heads=40, head_dim=128, rot=128, dtype="bf16", far=131071, transposed=True, **long),
        # a single request's new token
        dict(name="append 1x1", op="append", seqs=1, new_lo=1, new_hi=1, past_hi=511, far=0, heads=16, kv_heads=16, head_dim=64, page=16, rot=64, dtype="bf16", **plain),
        # a decode step of a batch behind a long shared context
        dict(name="append 256x1", op="append", seqs=256, new_lo=1, new_hi=1, past_hi=511, far=100000, heads=64, kv_heads=8, head_dim=128, page=64, rot=128, dtype="bf16", **long),
        # prompts of several requests, ragged, some behind an already cached part; half of each head rotated
        dict(name="append 6 prompts", op="append", seqs=6, new_lo=17, new_hi=4096, past_hi=300, far=0, heads=32, kv_heads=8, head_dim=128, page=64, rot=64, dtype="f16",
             **{**plain, "layout": "interleaved"}),
        # a few answers to a short prompt, no shared heads: latency
        dict(name="prefix 4 on 777", op="prefix", groups=1, seqs=4, pre_lo=777, pre_hi=777, own_lo=0, own_hi=60, heads=16, kv_heads=16, head_dim=64, page=16, dtype="bf16"),
        # a decode batch behind one system prompt
        dict(name="prefix 48 on 8k", op="prefix", groups=1, seqs=48, pre_lo=8192, pre_hi=8192, own_lo=1, own_hi=2048, heads=32, kv_heads=8, head_dim=128, page=64, dtype="bf16"),
        # several samples of each of several prompts, as reinforcement learning draws them
        dict(name="prefix 7 groups of 13", op="prefix", groups=7, seqs=91, pre_lo=211, pre_hi=6000, own_lo=0, own_hi=1024, heads=40, kv_heads=8, head_dim=128, page=32, dtype="f16"),
        # few questions to one very long document: bandwidth, split over the length
        dict(name="prefix 3 on 262k", op="prefix", groups=1, seqs=3, pre_lo=262143, pre_hi=262143, own_lo=17, own_hi=300, heads=64, kv_heads=8, head_dim=128, page=64, dtype="bf16"),
        # many answers behind a long context: products and exponentials bound
        dict(name="prefix 256 on 32k", op="prefix", groups=1, seqs=256, pre_lo=32768, pre_hi=32768, own_lo=1, own_hi=512, heads=64, kv_heads=8, head_dim=128, page=64, dtype="bf16"),
    ]


def log_int(rng, lo, hi):
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return n


def draw(rng):
    op = rng.choice(["rope", "append", "prefix", "prefix"])
    angles = dict(layout=rng.choice(["half", "interleaved"]), base=rng.choice([10000.0, 500000.0]), scaling=rng.choice(["none", "linear", "base", "parts"]), original=8192)
    angles["factor"] = 1.0 if angles["scaling"] == "none" else rng.choice([2.0, 8.0, 32.0])
    angles["amplitude"] = rng.choice([1.0, 1.0, 1.1386])
    if op == "rope":
        head_dim = rng.choice([64, 128, 128, 96, 80, 2 * rng.randint(9, 64)])      # heads too that start unaligned
        rot = rng.choice([head_dim, head_dim, head_dim // 4 * 2, max(2, head_dim // 8 * 2)])
        heads = rng.choice([1, 5, 8, 16, 25, 32, 64])
        return dict(op=op, tokens=log_int(rng, 1, max(1, (1 << 25) // (heads * head_dim))), heads=heads, head_dim=head_dim, rot=rot, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    far=rng.choice([4095, 131071, 1048575]), transposed=rng.random() < 0.4, **angles)
    if op == "append":
        new, head_dim, kv_heads = log_int(rng, 1, 2048), rng.choice([64, 128]), rng.choice([1, 2, 4, 8, 16])
        return dict(op=op, seqs=log_int(rng, 1, max(1, min(256, 8192 // new))), new_lo=rng.choice([0, 1, new]), new_hi=new, past_hi=rng.choice([0, 63, 511]),
                    far=rng.choice([0, 0, 100000]), heads=kv_heads * rng.choice([1, 3, 4]), kv_heads=kv_heads, head_dim=head_dim, page=rng.choice([16, 32, 64, 128]),
                    rot=rng.choice([head_dim, head_dim, head_dim // 2, 16]), dtype=rng.choice(["bf16", "bf16", "f16"]), **angles)
    kv_heads, head_dim = rng.choice([1, 2, 4, 8, 16]), rng.choice([64, 128])
    heads = kv_heads * rng.choice([1, 2, 4, 5, 8, 16])
    top = log_int(rng, 16, 131072)
    seqs = log_int(rng, 2, max(2, min(256, MOST // (top * heads))))
    groups = rng.choice([1, 1, 1, min(seqs, 2), min(seqs, 5), min(seqs, 16)])
    while groups > 1 and groups * top * kv_heads * head_dim * 2 > 1 << 28:
        groups -= 1
    own_hi = log_int(rng, 1, max(1, min(4096, (1 << 27) // (seqs * kv_heads * head_dim * 2))))
    return dict(op=op, groups=groups, seqs=seqs, pre_lo=rng.choice([0, 1, top]), pre_hi=top, own_lo=rng.choice([0, 1, own_hi]), own_hi=own_hi, heads=heads, kv_heads=kv_heads,
                head_dim=head_dim, page=rng.choice([16, 32, 64, 128]), dtype=rng.choice(["bf16", "bf16", "f16"]))


# ------------------------------------------------------------------ shapes that follow from a case
def spread(n, lo, hi, shift=0.0):
    """n whole numbers in [lo, hi], evenly but irregularly spread, the first at the upper end."""
    return [hi - int(((i * 0.6180339887498949 + shift) % 1.0) * (hi - lo + 1)) if hi > lo else hi for i in range(n)]


def append_shape(c):
    new = spread(c["seqs"], c["new_lo"], c["new_hi"])
    past = spread(c["seqs"], 0, c["past_hi"], 0.25)
    cols = max(-(-(p + n) // c["page"]) for p, n in zip(past, new)) + 1
    return new, past, cols


def prefix_shape(c):
    """Prefix lengths, first sequence of each group (and the end), own lengths."""
    first = [c["seqs"] * g // c["groups"] for g in range(c["groups"] + 1)]
    return spread(c["groups"], c["pre_lo"], c["pre_hi"]), first, spread(c["seqs"], c["own_lo"], c["own_hi"], 0.4)


def work(case):
    c = case
    if c["op"] == "rope":
        n = c["tokens"] * c["heads"] * c["head_dim"]
        return {"bytes": 2 * n * BYTES[c["dtype"]] + 4 * c["tokens"], "flops": 3 * c["tokens"] * c["heads"] * c["rot"]}
    if c["op"] == "append":
        tok, d = sum(append_shape(c)[0]), c["head_dim"]
        return {"bytes": tok * d * (4 * c["heads"] + 6 * c["kv_heads"]), "flops": tok * (3 * c["rot"] * (c["heads"] + c["kv_heads"]) + 4 * d * c["kv_heads"])}
    pre, first, mine = prefix_shape(c)
    d, nkv = c["head_dim"], c["kv_heads"]
    cached = sum(pre) + sum(mine)
    seen = sum(mine) + sum(p * (b - a) for p, a, b in zip(pre, first, first[1:]))
    pages = sum(-(-n // c["page"]) for n in pre + mine)
    return {"bytes": cached * nkv * d * 2 + pages * nkv * 8 + 4 * c["seqs"] * c["heads"] * (d + 1), "flops": 4 * seen * c["heads"] * d}


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

    def int32(values):
        return torch.tensor(values, dtype=torch.int32, device=DEV)

    s = dict(c)
    d, dt = c["head_dim"], DTYPES[c["dtype"]]
    if c["op"] == "rope":
        s["x"] = normal(c["tokens"], c["heads"], d, dtype=dt)
        # a batch's tokens: runs of neighbouring positions that start anywhere
        start = torch.randint(0, c["far"] + 1, (-(-c["tokens"] // 512),), generator=g, device=DEV)
        s["positions"] = ((start[:, None] + torch.arange(512, device=DEV)).flatten()[:c["tokens"]] % (c["far"] + 1)).to(torch.int32)
    else:
        if c["op"] == "append":
            new, lens, cols = append_shape(c)
            total = sum(new)
            s["cu_new"] = int32([sum(new[:i]) for i in range(c["seqs"] + 1)])
            s["max_new"] = max(new)
            s["q"] = normal(total, c["heads"], d, dtype=dt)
            s["k"], s["v"] = (normal(total, c["kv_heads"], d, std=w, dtype=dt) for w in (2.0, 0.7))
            # behind a shared prefix of `far` tokens, which the sequences' own lengths do not count
            s["positions"] = int32([c["far"] + p + j for p, n in zip(lens, new) for j in range(n)]) if c["far"] else None
            n_pages = c["seqs"] * cols + 3
        else:
            pre, first, lens = prefix_shape(c)
            cols, pre_cols = (max(1, -(-max(n) // c["page"])) for n in (lens, pre))
            n_pages = c["seqs"] * cols + c["groups"] * pre_cols + 3
            s["query"] = normal(c["seqs"], c["heads"], d, dtype=dt)
            s["sm_scale"] = 1.0 / math.sqrt(d)
            s["prefix_lengths"], s["cu_seqs"] = int32(pre), int32(first)
        order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        s["table"] = order[:c["seqs"] * cols].reshape(c["seqs"], cols).contiguous()
        if c["op"] == "prefix":
            s["prefix_table"] = order[c["seqs"] * cols:c["seqs"] * cols + c["groups"] * pre_cols].reshape(c["groups"], pre_cols).contiguous()
        s["lengths"] = int32(lens)
        shape = (n_pages, c["kv_heads"], c["page"], d)
        s["k_cache"], s["v_cache"] = bytes8(*shape), bytes8(*shape)
        # powers of two, as the append writes them
        s["k_scale"], s["v_scale"] = (torch.exp2(torch.randint(lo, lo + 3, shape[:2], generator=g, device=DEV).float()) for lo in (-8, -9))
    if own and c["op"] != "prefix":      # a program makes its frequencies once
        from paper_2607_18631_b200 import ops
        s["rotary"] = ops.Rotary(c["rot"], layout=c["layout"], base=c["base"], scaling=c["scaling"], factor=c["factor"], original=c["original"], amplitude=c["amplitude"])
    return s


# ------------------------------------------------------------------ one pass
def run(state):
    s = state
    if own:
        from paper_2607_18631_b200 import ops
        cache = [s.get(n) for n in ("k_cache", "v_cache", "k_scale", "v_scale")]
        if s["op"] == "rope":
            return ops.pf_rope(s["x"], s["positions"], s["rotary"], transposed=s["transposed"])
        if s["op"] == "append":
            q = ops.pf_kv_append_rope(*cache, s["q"], s["k"], s["v"], s["cu_new"], s["lengths"], s["table"], s["rotary"], max_new=s["max_new"], positions=s["positions"])
            return {"q": q, **{n: s[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale")}}
        return ops.pf_prefix_attention(s["query"], *cache, s["lengths"], s["table"], s["prefix_lengths"], s["prefix_table"], s["cu_seqs"], sm_scale=s["sm_scale"], lse=True)
    return {"rope": plain_rope, "append": plain_append, "prefix": plain_prefix}[s["op"]](s)


def frequencies(c):
    """Radians a position, in 64 bits."""
    i = torch.arange(c["rot"] // 2, dtype=torch.float64, device=DEV)
    base = c["base"] * (c["factor"] ** (c["rot"] / (c["rot"] - 2)) if c["scaling"] == "base" and c["rot"] > 2 else 1.0)
    f = base ** (-2.0 * i / c["rot"])
    if c["scaling"] == "linear":
        f = f / c["factor"]
    if c["scaling"] == "parts":      # pairs that turn often within the original context stay, those that hardly turn are stretched
        ramp = ((c["original"] * f / (2.0 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
        f = f * (ramp + (1.0 - ramp) / c["factor"])
    return f


def rotated(x, positions, c, transposed=False):
    """x: [tokens, heads, head_dim], in 32 bits."""
    angle = positions.double()[:, None] * frequencies(c)
    cos, sin = ((t * c["amplitude"]).float()[:, None, :] for t in (torch.cos(angle), torch.sin(angle)))
    if transposed:
        sin = -sin
    x, R = x.float(), c["rot"]
    out = x.clone()
    one, two = (slice(0, R // 2), slice(R // 2, R)) if c["layout"] == "half" else (slice(0, R, 2), slice(1, R, 2))
    out[..., one] = x[..., one] * cos - x[..., two] * sin
    out[..., two] = x[..., two] * cos + x[..., one] * sin
    return out


def plain_rope(s):
    return rotated(s["x"], s["positions"], s, s["transposed"]).to(s["x"].dtype)


def pow2_scale(amax):
    """The least power of two that brings amax into the 8-bit range, 2^-100 at least."""
    m, e = torch.frexp(amax)
    e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.ldexp(torch.ones_like(amax), torch.where(amax > 0, e, -100).clamp(-100, 118))


def plain_append(s):
    P = s["page"]
    cu, lens, table = s["cu_new"].long(), s["lengths"].long(), s["table"].long()
    n_new, total = cu[1:] - cu[:-1], s["k"].shape[0]
    seq = torch.repeat_interleave(torch.arange(s["seqs"], device=DEV), n_new, output_size=total)
    pos = lens[seq] + torch.arange(total, device=DEV) - cu[seq]
    angle_at = pos if s["positions"] is None else s["positions"]
    q, k = rotated(s["q"], angle_at, s).to(s["q"].dtype), rotated(s["k"], angle_at, s)
    page, slot = table[seq, pos // P], pos % P
    # the only page of a sequence that can hold earlier tokens is the one its first new token falls into
    head = table.gather(1, (lens // P).clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    before = torch.where(n_new > 0, lens % P, 0)
    kept = (torch.arange(P, device=DEV)[None, :] < before[:, None])[:, None, :, None]
    for cache, scale, x in ((s["k_cache"], s["k_scale"], k), (s["v_cache"], s["v_scale"], s["v"].float())):
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
    return {"q": q, **{n: s[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale")}}


def plain_prefix(s):
    B, nh, d = s["query"].shape
    nkv, P, G = s["kv_heads"], s["page"], nh // s["kv_heads"]
    q = s["query"].float().reshape(B, nkv, G, d)

    def dense(name, table):
        at = table.long()
        x = s[name + "_cache"].view(torch.uint8)[at].view(F8).float() * s[name + "_scale"][at][..., None, None]      # [n, cols, nkv, P, d]
        return x.permute(0, 2, 1, 3, 4).reshape(at.shape[0], nkv, at.shape[1] * P, d)

    def part(q, table, lengths):
        """q: [n, nkv, rows, d]; largest score, sum and weighted values of each row over its table's tokens."""
        score = torch.matmul(q, dense("k", table).transpose(2, 3)) * s["sm_scale"]
        seen = torch.arange(score.shape[-1], device=DEV)[None, :] < lengths.long()[:, None]
        score = score.masked_fill(~seen[:, None, None, :], float("-inf"))
        top = score.amax(-1, keepdim=True)
        e = torch.exp(score - torch.where(top == float("-inf"), 0.0, top))
        return top, e.sum(-1, keepdim=True), torch.matmul(e, dense("v", table))

    top, total, values = part(q, s["table"], s["lengths"])
    _, first, _ = prefix_shape(s)
    shared = []
    for g in range(s["groups"]):
        a, b = first[g], first[g + 1]
        rows = q[a:b].permute(1, 0, 2, 3).reshape(1, nkv, (b - a) * G, d)
        shared.append([t.reshape(nkv, b - a, G, -1).permute(1, 0, 2, 3) for t in part(rows, s["prefix_table"][g:g + 1], s["prefix_lengths"][g:g + 1])])
    p_top, p_total, p_values = (torch.cat([x[i] for x in shared]) for i in range(3))
    most = torch.maximum(top, p_top)
    z = torch.where(most == float("-inf"), 0.0, most)
    mine, theirs = torch.exp(top - z), torch.exp(p_top - z)
    total = total * mine + p_total * theirs
    out = (values * mine + p_values * theirs) / torch.where(total > 0, total, 1.0)
    return {"out": out.reshape(B, nh, d).to(s["query"].dtype), "lse": (z + torch.log(total)).reshape(B, nh)}


# ------------------------------------------------------------------ 64-bit values
def exact(case, seed):
    """What `run` returns, from the definitions in 64 bits; 8-bit outputs before their rounding."""
    c = case
    s = prepare(c, seed)
    f64 = torch.float64

    def turn(x, positions, sign=1.0):
        """Pairs as complex numbers, multiplied by amplitude * exp(i * angle)."""
        R, pairs = c["rot"], []
        base = c["base"]
        if c["scaling"] == "base" and R > 2:
            base *= c["factor"] ** (R / (R - 2))
        for i in range(R // 2):
            f = base ** (-2.0 * i / R)
            if c["scaling"] == "linear":
                f /= c["factor"]
            elif c["scaling"] == "parts":
                keep = min(1.0, max(0.0, (c["original"] * f / (2.0 * math.pi) - 1.0) / 31.0))
                f = keep * f + (1.0 - keep) * f / c["factor"]
            pairs.append(f)
        angle = positions.to(f64).unsqueeze(1) * torch.tensor(pairs, dtype=f64, device=DEV).unsqueeze(0)
        unit = torch.polar(torch.full_like(angle, c["amplitude"]), sign * angle).unsqueeze(1)
        x = x.to(f64)
        if c["layout"] == "half":
            z = torch.complex(x[:, :, :R // 2].contiguous(), x[:, :, R // 2:R].contiguous()) * unit
            head = torch.cat([z.real, z.imag], 2)
        else:
            head = torch.view_as_real(torch.view_as_complex(x[:, :, :R].unflatten(2, (R // 2, 2)).contiguous()) * unit).flatten(2)
        return torch.cat([head, x[:, :, R:]], 2)

    if c["op"] == "rope":
        return turn(s["x"], s["positions"], -1.0 if c["transposed"] else 1.0)
    if c["op"] == "append":
        new, past, _ = append_shape(c)
        at = s["positions"]
        if at is None:
            at = torch.tensor([p + j for p, n in zip(past, new) for j in range(n)], device=DEV)
        out = {"q": turn(s["q"], at)}
        table, P, done = s["table"].tolist(), c["page"], 0
        rows = []          # (page, first slot, last slot, first token of k / v)
        for b, (n, p) in enumerate(zip(new, past)):
            j = 0
            while j < n:
                slot = (p + j) % P
                m = min(P - slot, n - j)
                rows.append((table[b][(p + j) // P], slot, slot + m, done + j))
                j += m
            done += n
        for name, x in (("k", turn(s["k"], at)), ("v", s["v"].to(f64))):
            values, scale = s[name + "_cache"].to(f64), s[name + "_scale"].to(f64)
            for page, lo, hi, t in rows:
                part = x[t:t + hi - lo].transpose(0, 1)                                       # [heads, tokens, head_dim]
                need = torch.exp2(torch.ceil(torch.log2(part.abs().amax((1, 2)) / F8_MAX) - 1e-9))   # 7.0 / 448 is a power of two
                now = torch.maximum(need, scale[page]) if lo else need
                values[page, :, :lo] *= (scale[page] / now)[:, None, None]
                values[page, :, lo:hi] = part / now[:, None, None]
                scale[page] = now
            out[name + "_cache"], out[name + "_scale"] = values, scale
        return out
    pre, first, lens = prefix_shape(c)
    G, d = c["heads"] // c["kv_heads"], c["head_dim"]
    out = torch.zeros(c["seqs"], c["heads"], d, dtype=f64, device=DEV)
    lse = torch.full((c["seqs"], c["heads"]), float("-inf"), dtype=f64, device=DEV)

    def tokens(name, h, row, n):
        pages = row[:-(-n // c["page"])].long()
        return (s[name + "_cache"][:, h].view(torch.uint8)[pages].view(F8).to(f64) * s[name + "_scale"][pages, h].to(f64)[:, None, None]).reshape(-1, d)[:n]

    for g, n in enumerate(pre):
        for h in range(c["kv_heads"]):
            k0, v0 = (tokens(m, h, s["prefix_table"][g], n) for m in ("k", "v"))
            for b in range(first[g], first[g + 1]):
                if n + lens[b] == 0:
                    continue
                k, v = (torch.cat([x, tokens(m, h, s["table"][b], lens[b])]) for m, x in (("k", k0), ("v", v0)))
                score = s["query"][b, h * G:(h + 1) * G].to(f64) @ k.T * s["sm_scale"]
                lse[b, h * G:(h + 1) * G] = torch.logsumexp(score, -1)
                out[b, h * G:(h + 1) * G] = torch.softmax(score, -1) @ v
    return {"out": out, "lse": lse}
