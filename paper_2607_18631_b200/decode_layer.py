"""One decode layer of a ranked serving plan, run on this GPU: what the plan's per-layer step time is made of.

The serving model prices a decode step per layer as the attention (projection weights and cached keys and values over
HBM) plus the experts (the weights of those that a token chose).  `DecodeLayer` holds one layer as one GPU of a plan
holds it -- attention heads over tp, experts over ep, expert width over what is left -- with random weights, and runs
its step with the operators of `ops`; the projections are plain matrix products.  `measure` times the parts out of HBM, and
`with_measured_hbm` puts the rate they reached into a plan space's cluster, so that the space is ranked again with it.
(The model's other measured numbers, the efficiencies by tokens an expert, stay as they are.)

    python -m paper_2607_18631_b200.decode_layer [--batch N] [--context N] [--prefix N] [--rope BASE]

With `rotary`, queries and keys are rotated to their positions; with `prefix`, all sequences share that many tokens in front of their own.

Plans with latent attention (attn_kind 1) are refused: the cache here holds keys and values per head.  Collectives
between the GPUs of a plan are not run (a step's results are this GPU's parts).
"""
from __future__ import annotations

import argparse
import copy

from .binding import PF_ECUDA, PF_EINVAL, PlanfrontError

CAP_SLACK = 64       # tokens a sequence may grow by after the context it starts with
MIN_RATE_BYTES = 32_000_000   # 5 us at HBM's rate: what less takes is mostly launches and dependent reads


def layer_shape(cfg: dict, plan: dict) -> dict:
    """What one GPU of a serving plan (a decoded tuple: kv, batch, dpa, ep, tp) holds of a layer, and the tokens of a step.

    tokens: sequences whose attention runs here.  expert_tokens: tokens that the experts here see: with data-parallel attention those of
    all ep groups, as the serving model counts them.  Shared experts (`shared` of width `shared_ffn`) are split over tp like the rest of
    the dense weights and see this GPU's own tokens."""
    m, k = cfg["model"], cfg["kern"][plan["kv"]]
    tp, ep, batch = plan["tp"], plan["ep"], plan["batch"]

    def refuse(why):
        raise PlanfrontError(PF_EINVAL, f"decode_layer: {why}")
    if m["attn_kind"] != 0:
        refuse("latent attention has no per-head cache")
    if m["nh"] % tp or m["E"] % ep or m["nkv"] < 1:
        refuse("heads do not divide by tp, or experts by ep")
    if m["nkv"] % tp and tp % m["nkv"]:
        refuse(f"{m['nkv']} key / value heads cannot be split over tp {tp}")
    tokens = batch // ep if plan["dpa"] else batch
    if tokens < 1:
        refuse(f"a batch of {batch} leaves GPUs of ep {ep} without a sequence")
    engine = tp * ep if plan["dpa"] else tp          # GPUs of one engine, as the serving model counts them
    moe_tp = max(1, engine // ep)
    return dict(tokens=tokens, expert_tokens=batch, hidden=m["H"], heads=m["nh"] // tp, kv_heads=max(1, m["nkv"] // tp), head_dim=m["hd"],
                experts=m["E"], local=m["E"] // ep, top_k=m["K"], ffn=-(-m["F"] // moe_tp), shared=m["S"], shared_ffn=-(-m["Fs"] // tp) if m["S"] else 0,
                weights="e4m3" if k["wbytes"] == 1 else "bf16")


class DecodeLayer:
    """A layer's weights and cache on the current device, and its decode step.  shape: see layer_shape (expert_tokens, if left out, is
    tokens, and shared_ffn is ffn); context: cached tokens of every sequence at the start; prefix: tokens in front of them that all sequences share;
    rotary: arguments of ops.Rotary, its `rot` among them."""

    def __init__(self, shape: dict, context: int, page: int = 64, seed: int = 0, prefix: int = 0, rotary: dict | None = None):
        import torch

        from . import ops
        self.ops, self.torch, self.shape = ops, torch, dict(shape)
        s, dev = self.shape, torch.device("cuda", torch.cuda.current_device())
        g = torch.Generator(device=dev).manual_seed(seed)
        H, d, nh, nkv, T = s["hidden"], s["head_dim"], s["heads"], s["kv_heads"], s["tokens"]

        def weight(*dims):
            return (torch.randn(*dims, generator=g, device=dev) * dims[-1] ** -0.5).to(torch.bfloat16)

        self.norm1, self.norm2 = (torch.ones(H, dtype=torch.bfloat16, device=dev) for _ in range(2))
        self.w_qkv, self.w_out = weight((nh + 2 * nkv) * d, H), weight(H, nh * d)
        s.setdefault("expert_tokens", T)
        s.setdefault("shared_ffn", s["ffn"])
        self.router = None

        def layer_of(n, ffn, n_shared):
            mats, scales = [], [None] * 3
            for i, dims in enumerate(((n, ffn, H), (n, ffn, H), (n, H, ffn))):
                if s["weights"] == "bf16":
                    mats.append(torch.cat([weight(1, *dims[1:]) for _ in range(n)]))
                    continue
                mats.append(torch.cat([(torch.randn(1, *dims[1:], generator=g, device=dev) * 112).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
                                       for _ in range(n)]).view(torch.float8_e4m3fn))
                scales[i] = torch.full((n, -(-dims[1] // 128), -(-dims[2] // 128)), dims[2] ** -0.5 / 112, device=dev)
            if self.router is None:
                self.router = weight(s["experts"], H)
            return ops.MoeLayer(self.router, *mats, top_k=s["top_k"], n_shared=n_shared, gate_scale=scales[0], up_scale=scales[1], down_scale=scales[2])

        # shared experts go with the routed ones where they have the same width and tokens, else they are a layer of their own
        together = not s["shared"] or (s["shared_ffn"] == s["ffn"] and s["expert_tokens"] == T)
        self.moe = layer_of(s["local"] + (s["shared"] if together else 0), s["ffn"], s["shared"] if together else 0)
        self.shared = None if together else layer_of(s["shared"], s["shared_ffn"], s["shared"])
        self.status = torch.zeros(3, dtype=torch.int32, device=dev)        # of the latest calls of the two layers of experts and of the attention
        # the other GPUs' tokens, which an all-gather would bring: they stay the same from step to step
        others = torch.randn(s["expert_tokens"] - T, H, generator=g, device=dev).to(torch.bfloat16)
        self.others = ops.pf_add_rms_norm(others, None, self.norm2, y=True) if others.shape[0] else None
        cols = -(-(context + CAP_SLACK) // page)
        self.table = torch.randperm(T * cols, generator=g, device=dev).to(torch.int32).reshape(T, cols)
        if prefix < 0:
            raise PlanfrontError(PF_EINVAL, f"decode_layer: a prefix of {prefix} tokens")
        prefix_pages = -(-prefix // page)
        self.cache = [torch.empty(T * cols + prefix_pages, nkv, page, d, dtype=torch.float8_e4m3fn, device=dev) for _ in range(2)]
        self.scales = [torch.empty(T * cols + prefix_pages, nkv, device=dev) for _ in range(2)]
        self.rotary = None if rotary is None else ops.Rotary(**rotary)
        self.prefix = prefix
        self.lengths = torch.zeros(T, dtype=torch.int32, device=dev)
        self.one_each = torch.arange(T + 1, dtype=torch.int32, device=dev)
        self.room = cols * page

        def prompt(n, seqs, lengths, table, first):         # in chunks, as a prefill appends it
            at = 0
            while at < n:
                m = min(n - at, 1024)
                k, v = (torch.randn(seqs * m, nkv, d, generator=g, device=dev).to(torch.bfloat16) for _ in range(2))
                self.append(None, k, v, self.one_each[:seqs + 1] * m, lengths, table, m, (lengths[:, None] + torch.arange(first, first + m, device=dev)).flatten().int())
                lengths += m
                at += m

        prompt(context, T, self.lengths, self.table, prefix)
        if prefix:
            self.prefix_table = torch.arange(T * cols, T * cols + prefix_pages, dtype=torch.int32, device=dev)[None]
            self.prefix_length = torch.zeros(1, dtype=torch.int32, device=dev)
            prompt(prefix, 1, self.prefix_length, self.prefix_table, 0)
        self.cached = context

    def append(self, q, k, v, cu_new, lengths, table, max_new, positions):
        """New keys and values into the cache, rotated to `positions` where the layer does so; returns the queries, rotated likewise."""
        if self.rotary is None:
            self.ops.pf_kv_append(*self.cache, *self.scales, k, v, cu_new, lengths, table, max_new=max_new)
            return q
        return self.ops.pf_kv_append_rope(*self.cache, *self.scales, q, k, v, cu_new, lengths, table, self.rotary, max_new=max_new, positions=positions)

    def step(self, x, residual):
        """One token of every sequence through the layer: x is what the layer before added, residual the stream it adds to (updated
        in place).  Returns what this layer adds; the sequences are one token longer."""
        ops, s = self.ops, self.shape
        if self.cached >= self.room:
            raise PlanfrontError(PF_EINVAL, "decode_layer: the cache is full")
        y = ops.pf_add_rms_norm(x, residual, self.norm1, y=True, q=False, sum_out=residual)["y"]
        q, k, v = self.project(y)
        q = self.append(q, k, v, self.one_each, self.lengths, self.table, 1, self.lengths + self.prefix if self.prefix and self.rotary else None)
        self.lengths += 1
        self.cached += 1
        a = self.attend(q)
        n = ops.pf_add_rms_norm(a.flatten(1) @ self.w_out.t(), residual, self.norm2, y=True, sum_out=residual)
        return self.experts(n)

    def project(self, y):
        s = self.shape
        qkv = (y @ self.w_qkv.t()).unflatten(1, (s["heads"] + 2 * s["kv_heads"], s["head_dim"]))
        return qkv.split((s["heads"], s["kv_heads"], s["kv_heads"]), 1)

    def attend(self, q):
        if self.prefix:
            return self.ops.pf_prefix_attention(q, *self.cache, *self.scales, self.lengths, self.table, self.prefix_length, self.prefix_table,
                                                status=self.status[2:3])["out"]
        return self.ops.pf_decode_attention(q, *self.cache, *self.scales, self.lengths, self.table)["out"]

    def gather(self, n):
        """The tokens that the experts here see: this GPU's first, then the others'."""
        if self.others is None:
            return n
        whole = {k: self.torch.cat([n[k], self.others[k]]) for k in ("y", "scale")}
        whole["q"] = self.torch.cat([t["q"].view(self.torch.uint8) for t in (n, self.others)]).view(n["q"].dtype)
        return whole

    def run(self, layer, n, status):
        eight = (n["q"], n["scale"]) if self.shape["weights"] == "e4m3" else ()
        return layer.forward(n["y"], *eight, status=self.status[status:status + 1])["out"]

    def experts(self, n):
        out = self.run(self.moe, self.gather(n), 0)[:n["y"].shape[0]]
        return out if self.shared is None else out + self.run(self.shared, n, 1)

    def check(self):
        """Waits for the device; raises if a wait inside the experts' or the attention's latest call ran out (its output is NaN then)."""
        *experts, attention = self.status.tolist()
        if any(experts):
            raise PlanfrontError(PF_ECUDA, "decode_layer: a wait inside the experts' kernel ran out")
        if attention:
            raise PlanfrontError(PF_ECUDA, "decode_layer: a wait inside the kernel for shared prefixes ran out")

    def measure(self, repeats: int = 20) -> dict:
        """{part: (microseconds, bytes it cannot do without)} of the attention and the experts, device time of a call whose cache and weights
        come from HBM: in front of each, a buffer of four times the L2 is read."""
        torch, s = self.torch, self.shape
        x = torch.randn(s["tokens"], s["hidden"], device="cuda").to(torch.bfloat16)
        n = self.ops.pf_add_rms_norm(x, None, self.norm2, y=True)
        whole = self.gather(n)
        q = self.project(x)[0].contiguous()
        ids = self.moe.forward(whole["y"])["ids"]
        touched = int(torch.unique(ids[ids < s["local"]]).numel())
        element = 1 if s["weights"] == "e4m3" else 2
        cache_bytes = (int(self.lengths.sum()) + self.prefix) * s["kv_heads"] * s["head_dim"] * 2
        expert_bytes = 3 * s["hidden"] * (touched * s["ffn"] + s["shared"] * s["shared_ffn"]) * element

        def experts():
            self.run(self.moe, whole, 0)
            if self.shared is not None:
                self.run(self.shared, n, 1)
        evict = torch.zeros(torch.cuda.get_device_properties(x.device).L2_cache_size, dtype=torch.float32, device=x.device)
        out = {}
        for name, call, size in (("attention", lambda: self.attend(q), cache_bytes), ("experts", experts, expert_bytes)):
            call()
            events = [[torch.cuda.Event(enable_timing=True) for _ in range(2)] for _ in range(repeats)]
            for a, b in events:
                evict.amax()               # long enough for the host to have the call enqueued
                a.record()
                call()
                b.record()
            torch.cuda.synchronize()
            out[name] = (sum(a.elapsed_time(b) for a, b in events) * 1e3 / repeats, size)
        self.check()
        return out


def with_measured_hbm(cfg: dict, parts: dict) -> dict:
    """The plan space with the HBM rate that the measured parts reached together.  Parts of less than MIN_RATE_BYTES measure latency, not a rate, and
    do not count; without any other the rate stays as it is."""
    new = copy.deepcopy(cfg)
    large = [part for part in parts.values() if part[1] >= MIN_RATE_BYTES]
    if large:
        new["cluster"]["hbm_bw"] = sum(size for _, size in large) / (sum(us for us, _ in large) * 1e-6)
    return new


def example_space(batch: int, context: int) -> dict:
    """A small serving space of a model with grouped key / value heads: 6 of 64 experts, bf16 and e4m3 kernels, up to 8 GPUs."""
    kern = [dict(needs_caps=1 if fp8 else 0, avail_mask=0xFF, is_native=1, wbytes=1 if fp8 else 2, dtype_mult=2.0 if fp8 else 1.0, eff=[0.5] * 8, patch_ovh=0.0,
                 dtype=int(fp8)) for fp8 in (False, True)]
    return dict(
        name="decode-layer example", phase=1,
        model=dict(L=24, H=4096, nh=32, nkv=8, hd=128, attn_kind=0, E=64, K=6, F=1408, S=2, Fs=1408, seq=4096, vocab=102400, wb=2, gb=4, ob=12, ab=1, n_mats=3,
                   count_embeddings=1),
        cluster=dict(G=8, caps=1, budget_bytes=160_000_000_000, reserved_bytes=0, peak_flops=1.6e15, hbm_bw=7.7e12, bw_intra=770e9, bw_inter=50e9, alpha_intra=5e-6,
                     alpha_inter=10e-6),
        workload=dict(world=8, scen_P=[context], scen_O=[256]),
        consts=dict(eff_dense=0.6, bwd_factor=2.0, dp_overlap_frac=0.5, dualpipe_startup_div=8.0, step_overhead=1e-5),
        sched=[dict(kind=0, overlap=0, mapped=1, hide_frac=0.0, sched_ovh=0.0)], kern=kern,
        rules=dict(ep_scope=0, layer_mode=0, tp_max=8, world_min=1, world_max=8, enforce_realizability=1),
        axes=[("kv", [0, 1]), ("chunk", [1024, 4096]), ("batch", [batch]), ("dpa", [0]), ("ep", [1, 2, 4, 8]), ("tp", [1, 2, 4, 8]), ("scen", [0])])


def best_plan(cfg: dict):
    """(decoded tuple, predicted tokens/s/GPU) of the space's first plan."""
    import torch

    from .binding import Plan
    plan = Plan(cfg)
    out = plan.score(k=1)
    torch.cuda.synchronize()
    if int(out["topk_count"].item()) == 0:
        raise PlanfrontError(PF_EINVAL, "decode_layer: no feasible plan")
    best = plan.decode(int(out["topk_idx"][0].item())), float(out["topk_score"][0].item())
    plan.close()
    return best


def main(argv=None) -> None:
    import torch
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--context", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=4)
    ap.add_argument("--prefix", type=int, default=0, help="tokens in front of the context that all sequences share")
    ap.add_argument("--rope", type=float, default=0.0, metavar="BASE", help="rotate queries and keys, with frequencies of this base")
    a = ap.parse_args(argv)
    cfg = example_space(a.batch, a.context)
    plan, tput = best_plan(cfg)
    shape = layer_shape(cfg, plan)
    print(f"plan: tp {plan['tp']} ep {plan['ep']} kernel {shape['weights']} batch {plan['batch']}: predicted {tput:.1f} tokens/s/GPU")
    layer = DecodeLayer(shape, a.context, prefix=a.prefix, rotary=dict(rot=shape["head_dim"], base=a.rope) if a.rope else None)
    x = torch.randn(shape["tokens"], shape["hidden"], device="cuda").to(torch.bfloat16)
    residual = torch.zeros_like(x)
    for _ in range(a.steps):
        x = layer.step(x, residual)
    layer.check()
    parts = layer.measure()
    for name, (us, size) in parts.items():
        rate = f"{size / us / 1e6:6.2f} TB/s" if size >= MIN_RATE_BYTES else "(latency)"
        print(f"{name:10s} {us:9.1f} us  {size / 1e6:9.1f} MB  {rate}")
    if a.prefix:
        del parts["attention"]      # the model prices every sequence's whole context, so the rate of a shared one is not its rate
    again = with_measured_hbm(cfg, parts)
    plan, tput = best_plan(again)
    print(f"with {again['cluster']['hbm_bw'] / 1e12:.2f} TB/s: tp {plan['tp']} ep {plan['ep']}, predicted {tput:.1f} tokens/s/GPU")


if __name__ == "__main__":
    main()
