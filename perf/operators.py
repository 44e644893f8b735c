"""The operators beside the MUXQ layer, as cases that can be timed and compared.

  norm      h = R + scale * gate * post(Y), x = pre(h): what stands between two projections of a transformer block.  Y is the
            projection's result, R the residual stream, x the fp16 input of the next projection.  post and pre are a layer
            norm, a root-mean-square norm or nothing.
  adapters  Y = base + s * (X A^T) B^T with low-rank adapters (A, B, s) of the row's request, many requests in one batch;
            base is the shared projection's result.

`own` says whether run() computes the plain form in torch or calls the package."""
import math

import torch

own = False

_NORM = {"op": "norm", "residual": "f32", "block": "f16", "post": "none", "pre": "layer", "gate": "none", "gate_type": "f32",
         "sequences": 1, "scale": 1.0}
_ADAPT = {"op": "adapters", "slots": 8, "ranks": "16", "requests": 8, "bare": 0, "order": "runs", "out": "f16"}


def listed():
    return [
        # one new token through a block of the small width: residual add and layer norm, launch and latency count
        dict(_NORM, name="norm_step_1", tokens=1, width=768),
        # one decode step of sixteen sequences; the projection before left fp32, the stream is fp16, a gate per channel
        dict(_NORM, name="norm_step_16", tokens=16, width=1280, residual="f16", block="f32", pre="rms", gate="channel", scale=0.5),
        # a prompt of odd length, width no multiple of 64 or 128, norms on both sides of the block
        dict(_NORM, name="norm_prompt_1003", tokens=1003, width=1040, block="f32", post="rms", pre="rms", gate="channel", scale=0.7),
        # eight prompts of 1024 tokens at the small width, everything in fp16
        dict(_NORM, name="norm_8192", tokens=8192, width=768, residual="f16"),
        # the first norm of a wide model on a prompt: no block before it, nothing added
        dict(_NORM, name="norm_first_wide", tokens=2048, width=5120, block="none"),
        # the largest prompt batch: fp32 stream, norms on both sides, a gate for every token
        dict(_NORM, name="norm_16384_gated", tokens=16384, width=1280, post="rms", pre="rms", gate="row", gate_type="f16", scale=0.5),
        # one new token of one request
        dict(_ADAPT, name="adapt_step_1", tokens=1, K=768, N=768, slots=1, ranks="8", requests=1),
        # one decode step of sixteen requests, an adapter each, in the order of the batch
        dict(_ADAPT, name="adapt_step_16", tokens=16, K=1280, N=3840, slots=16, requests=16, order="mixed"),
        # a mixed batch: sixty-one tokens of twenty-four requests, ranks of all sizes, a third of the requests without an adapter
        dict(_ADAPT, name="adapt_ragged_61", tokens=61, K=1040, N=1560, slots=11, ranks="4,8,13,33,64", requests=24, bare=3, order="mixed", out="f32"),
        # five prompts together, odd lengths, fp32 results
        dict(_ADAPT, name="adapt_prompt_1003", tokens=1003, K=1280, N=5120, slots=5, ranks="16,32", requests=5, out="f32"),
        # eight prompts of 1024 tokens at the small width, every fourth without an adapter
        dict(_ADAPT, name="adapt_8192", tokens=8192, K=768, N=2304, slots=6, ranks="32", requests=8, bare=4),
        # the largest prompt batch at the large width and a high rank
        dict(_ADAPT, name="adapt_16384_rank64", tokens=16384, K=1280, N=5120, ranks="64", requests=16),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _fits(case):
    """No more than the largest listed case of the operator."""
    most = work(listed()[5] if case["op"] == "norm" else listed()[-1])
    w = work(case)
    return w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]


def draw(rng):
    while True:
        if rng.random() < 0.5:
            block = rng.choice(("f16", "f16", "f32", "none"))
            post = "none" if block == "none" else rng.choice(("none", "none", "rms", "layer"))
            gate = "none" if block == "none" else rng.choice(("none", "channel", "row", "sequence"))
            tokens = _log_uniform(rng, 1, 16384)
            sequences = rng.randint(1, min(tokens, 16)) if gate == "sequence" else 1
            case = dict(_NORM, tokens=tokens // sequences * sequences, width=8 * _log_uniform(rng, 8, 1024), residual=rng.choice(("f32", "f16")),
                        block=block, post=post, pre=rng.choice(("layer", "rms")), gate=gate, gate_type=rng.choice(("f16", "f32")),
                        sequences=sequences, scale=round(rng.uniform(0.2, 1.5), 3))
        else:
            tokens = _log_uniform(rng, 1, 16384)
            requests = rng.randint(1, min(tokens, 32)) if rng.random() < 0.7 else _log_uniform(rng, 1, min(tokens, 256))
            ranks = rng.choice(("8", "16", "16", "32", "64", "128", "%d" % rng.randint(1, 64), "4,8,13,33,64", "16,32", "8,16,100"))
            case = dict(_ADAPT, tokens=tokens, K=8 * _log_uniform(rng, 48, 640), N=8 * _log_uniform(rng, 48, 640),
                        slots=rng.randint(1, min(requests, 32)), ranks=ranks, requests=requests, bare=rng.choice((0, 0, 0, 2, 3, 5)),
                        order=rng.choice(("runs", "runs", "mixed")), out=rng.choice(("f16", "f16", "f32")))
        if _fits(case):
            return case


def _type(name):
    return torch.float32 if name == "f32" else torch.float16


def _ranks(case):
    given = [int(r) for r in case["ranks"].split(",")]
    return [given[i % len(given)] for i in range(case["slots"])]


def _slots(case):
    """The slot of every token, requests one after the other, their lengths as even as they come."""
    M, requests, bare = case["tokens"], case["requests"], case["bare"]
    out = []
    for j in range(requests):
        slot = -1 if bare and j % bare == bare - 1 else j % case["slots"]
        out += [slot] * ((j + 1) * M // requests - j * M // requests)
    return out


def _stream(gen, tokens, width, outliers=8):
    """Activations: N(0, 1) and a few channels that are 40 to 80 times as large."""
    x = torch.randn(tokens, width, device="cuda", generator=gen)
    channels = torch.randperm(width, device="cuda", generator=gen)[:outliers]
    x[:, channels] *= 40.0 + 40.0 * torch.rand(outliers, device="cuda", generator=gen)
    return x


def _vectors(gen, width):
    return 1.0 + 0.1 * torch.randn(width, device="cuda", generator=gen), 0.1 * torch.randn(width, device="cuda", generator=gen)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    M = case["tokens"]
    if case["op"] == "norm":
        D, kind = case["width"], _type(case["residual"])
        state = dict(case, R=_stream(gen, M, D).to(kind), Y=None, g=None, group=1, w_pre=None, b_pre=None, w_post=None, b_post=None,
                     X_out=torch.empty(M, D, dtype=torch.float16, device="cuda"), H_out=None)
        state["w_pre"], state["b_pre"] = _vectors(gen, D)
        state["w_post"], state["b_post"] = _vectors(gen, D)
        if case["block"] != "none":
            state["Y"] = torch.randn(M, D, device="cuda", generator=gen).to(_type(case["block"]))
            state["H_out"] = torch.empty(M, D, dtype=kind, device="cuda")
        if case["gate"] == "channel":
            state["g"] = 0.5 * torch.randn(D, device="cuda", generator=gen)
        elif case["gate"] != "none":
            rows = M if case["gate"] == "row" else case["sequences"]
            state["g"] = (0.5 * torch.randn(rows, D, device="cuda", generator=gen)).to(_type(case["gate_type"]))
            state["group"] = M // rows
        return state
    K, N, S, ranks = case["K"], case["N"], case["slots"], _ranks(case)
    most = (max(ranks) + 7) // 8 * 8  # room for the highest rank, in eights
    host = _slots(case)
    slot = torch.tensor(host, dtype=torch.int32, device="cuda")
    if case["order"] == "mixed":
        slot = slot[torch.randperm(M, device="cuda", generator=gen)]
    rank = torch.tensor(ranks, dtype=torch.int32, device="cuda")
    used = torch.arange(most, device="cuda")[None, :] < rank[:, None]
    A = torch.randn(S, most, K, device="cuda", generator=gen) / math.sqrt(K) * used[:, :, None]
    B = torch.randn(S, N, most, device="cuda", generator=gen) * 0.1 * used[:, None, :]
    kind = _type(case["out"])
    return dict(case, X=_stream(gen, M, K).half(), slot=slot, rank=rank, A=A.half(), B=B.half(),
                s=0.5 + torch.rand(S, device="cuda", generator=gen), base=torch.randn(M, N, device="cuda", generator=gen).to(kind),
                share=max(host.count(i) for i in set(host) - {-1}),  # the most tokens that any slot has: the scheduler's
                status=torch.zeros(1, dtype=torch.int32, device="cuda"), Y_out=torch.empty(M, N, dtype=kind, device="cuda"))


def _norm(v, kind, weight, bias):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(dim=1, keepdim=True)
    out = v / ((v * v).mean(dim=1, keepdim=True) + 1e-5).sqrt() * weight
    return out + bias if kind == "layer" else out


def _plain_norm(s):
    h = s["R"].float()
    if s["Y"] is not None:
        v = _norm(s["Y"].float(), s["post"], s["w_post"], s["b_post"])
        if s["g"] is not None:
            g = s["g"].float()
            v = v * (g if g.dim() == 1 else g.repeat_interleave(s["group"], dim=0, output_size=s["tokens"]))
        h = h + s["scale"] * v
    x = _norm(h, s["pre"], s["w_pre"], s["b_pre"]).half()
    return {"x": x} if s["Y"] is None else {"h": h.to(s["R"].dtype), "x": x}


def _plain_adapters(s):
    """Tokens sorted by slot, every slot's in a row of one batched product of each kind."""
    M, S, slot = s["tokens"], s["slots"], s["slot"].long()
    order = slot.argsort(stable=True)
    bounds = torch.searchsorted(slot[order], torch.arange(S + 1, device=slot.device))
    at = bounds[:-1, None] + torch.arange(s["share"], device=slot.device)[None, :]
    inside = at < bounds[1:, None]
    rows = order[at.clamp(max=M - 1)]
    keep = torch.arange(s["A"].shape[1], device=slot.device)[None, :] < s["rank"][:, None]
    t = torch.bmm(s["X"].float()[rows], s["A"].float().transpose(1, 2)) * keep[:, None, :]
    d = torch.bmm(t, s["B"].float().transpose(1, 2)) * s["s"][:, None, None]
    out = torch.cat([s["base"].float(), torch.zeros(1, s["N"], device=slot.device)])  # the last row takes what no token wants
    y = out.clone()
    y[torch.where(inside, rows, M)] = out[rows] + d
    return y[:M].to(s["base"].dtype)


def run(state):
    s = state
    if not own:
        return _plain_norm(s) if s["op"] == "norm" else _plain_adapters(s)
    import paper_2604_04701_b200 as mx
    if s["op"] == "adapters":
        return mx.muxq_adapters(s["X"], s["A"], s["B"], s["slot"], scale=s["s"], rank=s["rank"], base=s["base"], status=s["status"], out=s["Y_out"])
    kinds = {"none": mx.MUXQ_NORM_NONE, "rms": mx.MUXQ_NORM_RMS, "layer": mx.MUXQ_NORM_LAYER}
    pre = mx.Norm(kinds[s["pre"]], s["w_pre"], s["b_pre"] if s["pre"] == "layer" else None, 1e-5)
    if s["Y"] is None:
        return {"x": mx.muxq_residual_norm(s["R"], None, pre, X=s["X_out"])[1]}
    post = None if s["post"] == "none" else mx.Norm(kinds[s["post"]], s["w_post"], s["b_post"] if s["post"] == "layer" else None, 1e-5)
    h, x = mx.muxq_residual_norm(s["R"], s["Y"], pre, post=post, gate=s["g"], gate_group=s["group"], scale=s["scale"], H=s["H_out"], X=s["X_out"])
    return {"h": h, "x": x}


def work(case):
    """Inputs once, outputs once; of the adapters those that a token has."""
    M = case["tokens"]
    size = lambda name: {"f16": 2.0, "f32": 4.0, "none": 0.0}[name]  # noqa: E731
    if case["op"] == "norm":
        D = case["width"]
        r, y = size(case["residual"]), size(case["block"])
        rows = {"none": 0, "channel": 1, "row": M, "sequence": case["sequences"]}[case["gate"]]
        g = 4.0 if case["gate"] == "channel" else size(case["gate_type"])
        vectors = sum({"none": 0, "rms": 1, "layer": 2}[case[k]] for k in ("pre", "post"))
        flops = sum({"none": 0, "rms": 4, "layer": 7}[case[k]] for k in ("pre", "post")) + (2 if y else 0) + (1 if rows else 0)
        return {"bytes": M * D * (r + y + 2.0 + (r if y else 0.0)) + rows * D * g + 4.0 * vectors * D, "flops": float(flops) * M * D}
    K, N, ranks, slots = case["K"], case["N"], _ranks(case), _slots(case)
    out = size(case["out"])
    per_token = sum(2.0 * ranks[a] * (K + N) for a in slots if a >= 0)
    adapters = sum(2.0 * ranks[a] * (K + N) for a in set(slots) if a >= 0)
    return {"bytes": 2.0 * M * K + 2.0 * out * M * N + 4.0 * M + adapters, "flops": per_token + 2.0 * M * N}


def _exact_norm(v, kind, weight, bias):
    if kind == "none":
        return v
    mu = torch.sum(v, 1) / v.shape[1] if kind == "layer" else torch.zeros(v.shape[0], dtype=v.dtype, device=v.device)
    var = torch.einsum("md,md->m", v - mu[:, None], v - mu[:, None]) / v.shape[1]
    out = torch.einsum("md,m,d->md", v - mu[:, None], (var + 1e-5).pow(-0.5), weight.double())
    return out + bias.double() if kind == "layer" else out


def exact(case, seed):
    """The definitions in 64 bits: rows of the stream, and one request's tokens after the other."""
    s = prepare(case, seed)
    if case["op"] == "norm":
        h = s["R"].double()
        if s["Y"] is not None:
            v = _exact_norm(s["Y"].double(), case["post"], s["w_post"], s["b_post"])
            if s["g"] is not None:
                g = s["g"].double().reshape(-1, case["width"])
                v = (v.reshape(g.shape[0], -1, case["width"]) * g[:, None, :]).reshape(v.shape)
            h = h + case["scale"] * v
        x = _exact_norm(h, case["pre"], s["w_pre"], s["b_pre"])
        return {"x": x} if s["Y"] is None else {"h": h, "x": x}
    y = s["base"].double()
    for a in range(case["slots"]):
        mine, r = (s["slot"] == a).nonzero()[:, 0], int(s["rank"][a])
        down = torch.einsum("mk,rk->mr", s["X"][mine].double(), s["A"][a, :r].double())
        y[mine] += float(s["s"][a]) * torch.einsum("mr,nr->mn", down, s["B"][a, :, :r].double())
    return y
