"""Timed cases of linear attention with a decay, and of the norm around attention.

Linear attention keeps, per sequence and KV head, an FP32 state S [128][128] instead of a cache:
S_t = exp(g_t) S_{t-1} + k_t v_t^T and o_t = scale q_t^T S_t, where g <= 0 is the log decay of the
KV head, the same for all tokens or one per token.  Kinds:

  prefill  packed prompts, whole or chunks behind a state that an earlier call left;
  decode   one or a few new tokens per sequence behind its state;
  norm     root-mean-square norm of rows, with the residual's addition and E4M3 codes with scales
           (per row or per group of channels), or BF16 without.

States are read from some slots of a pool and left in others, as where drafted tokens may have to
be taken back.  Head shapes are the repository's (32:8, 40:8 and their four-way shards 8:2, 10:2)
and generic ones: one query head per KV head (8:8, 32:32), one KV head for all (16:1).
"""
import math

import torch

own = False

D = 128
DEV = "cuda"
EPS = 1e-6
SCALE = 1 / math.sqrt(D)


def listed():
    return [
        # one short user prompt, odd length: latency
        dict(name="prefill_777", kind="prefill", h_q=32, h_kv=8, new="777", carried=False, decay="head"),
        # four ragged user prompts that arrive together
        dict(name="prefill_prompts", kind="prefill", h_q=40, h_kv=8, new="1187,512,2049,300", carried=False, decay="head"),
        # a serving step's chunks on a four-way shard, behind the states that earlier chunks left
        dict(name="prefill_chunks", kind="prefill", h_q=8, h_kv=2, new="512,2048,1000,1", carried=True, decay="token"),
        # a document prompt, every head with keys of its own
        dict(name="prefill_8k", kind="prefill", h_q=32, h_kv=32, new="8192", carried=False, decay="token"),
        # one long document
        dict(name="prefill_64k", kind="prefill", h_q=32, h_kv=8, new="65536", carried=False, decay="head"),
        # one interactive sequence: the latency of a decode step's attention
        dict(name="decode_b1", kind="decode", h_q=32, h_kv=8, batch=1, rows=1, decay="head"),
        # a serving batch on a four-way shard
        dict(name="decode_b32", kind="decode", h_q=10, h_kv=2, batch=32, rows=1, decay="token"),
        # four drafted tokens verified at once
        dict(name="decode_b64_drafts", kind="decode", h_q=40, h_kv=8, batch=64, rows=4, decay="token"),
        # a large serving batch, every head with a state of its own
        dict(name="decode_b128", kind="decode", h_q=32, h_kv=32, batch=128, rows=1, decay="head"),
        # the residual stream before a projection in 8 bits, in a decode step
        dict(name="norm_step_b32", kind="norm", rows=32, width=4096, residual=True, out="row"),
        # the same for the tokens of long prompts, a scale per 128 channels
        dict(name="norm_16k", kind="norm", rows=16384, width=5120, residual=True, out="128"),
        # the heads' outputs of four prompts of 4048 tokens together, 40 heads each
        dict(name="norm_heads", kind="norm", rows=161920, width=128, residual=False, out="bf16"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["prefill", "decode", "norm"])
    if kind == "norm":
        width = 8 * log(1, 2048)
        return dict(kind=kind, rows=log(1, max(2, 16384 * 5120 // max(width, 256))), width=width, residual=rng.random() < 0.6,
                    out=rng.choice(["bf16", "row", "32", "64", "128", "256"]))
    h_q, h_kv = rng.choice([(32, 8), (40, 8), (8, 2), (10, 2), (8, 8), (16, 1), (32, 32)])
    decay = rng.choice(["head", "token"])
    if kind == "decode":
        return dict(kind=kind, h_q=h_q, h_kv=h_kv, batch=log(1, min(256, 4096 // h_kv)), rows=rng.choice([1, 1, 1, 2, 5, 8]), decay=decay)
    b = log(1, 32)
    most = min(65536, 65536 * 40 // (h_q + h_kv)) // b
    return dict(kind=kind, h_q=h_q, h_kv=h_kv, new=",".join(str(log(1, most)) for _ in range(b)), carried=rng.random() < 0.5, decay=decay)


# ---------------------------------------------------------------------------- inputs
def _lens(case):
    if case["kind"] == "decode":
        return [case["rows"]] * case["batch"]
    return [int(n) for n in case["new"].split(",")]


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case=case, kind=case["kind"])
    if s["kind"] == "norm":
        n, w = case["rows"], case["width"]
        eight = case["out"] != "bf16"
        group = w if case["out"] in ("row", "bf16") else int(case["out"])
        # a residual stream: a few channels much larger than the others
        size = torch.where(torch.rand(w, generator=gen, device=DEV) < 0.004, 30.0, 1.0)
        s.update(x=_normal(gen, n, w).to(torch.bfloat16), weight=(1 + 0.2 * _normal(gen, w)).to(torch.bfloat16), group=group,
                 residual=(_normal(gen, n, w) * size).to(torch.bfloat16) if case["residual"] else None,
                 residual_out=torch.empty(n, w, dtype=torch.bfloat16, device=DEV) if case["residual"] else None,
                 out=torch.empty(n, w, dtype=torch.float8_e4m3fn if eight else torch.bfloat16, device=DEV),
                 scales=torch.empty(n, -(-w // group), device=DEV) if eight else None)
        return s
    lens, h_q, h = _lens(case), case["h_q"], case["h_kv"]
    t, b = sum(lens), len(lens)
    carried = case.get("carried", True)
    if case["decay"] == "head":     # halves after 22 to 2800 tokens
        g = torch.log1p(-torch.pow(2.0, -5 - 7 * torch.arange(h, device=DEV) / h))
    else:                           # a gate per token: mostly near 1, some tokens that clear much of the state
        g = torch.nn.functional.logsigmoid(4 + 1.5 * _normal(gen, t, h))
    slots = torch.randperm(b * (2 if carried else 1), generator=torch.Generator().manual_seed(seed)).tolist()
    states = torch.zeros(len(slots), h, D, D, device=DEV)
    if carried:                     # what some hundred tokens left
        states[slots[b:]] = 4 * _normal(gen, b, h, D, D)
    s.update(q=_normal(gen, t, h_q, D).to(torch.bfloat16), k=_normal(gen, t, h, D).to(torch.bfloat16),
             v=_normal(gen, t, h, D).to(torch.bfloat16), g=g.float(), lens=lens, cu=_i32([sum(lens[:i]) for i in range(b + 1)]),
             states=states, dst=_i32(slots[:b]), src=_i32(slots[b:] if carried else [-1] * b),
             out=torch.empty(t, h_q, D, dtype=torch.bfloat16, device=DEV), workspace=None)
    if own and s["kind"] == "prefill":
        import paper_2609_33135_amd as mp
        size = mp.linear_prefill_workspace_size(b, t, max(lens), h_q, h)
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEV) if size else None
    return s


# ---------------------------------------------------------------------------- the framework's calls
def _run_own(s):
    import paper_2609_33135_amd as mp
    if s["kind"] == "norm":
        mp.rms_norm(s["x"], s["weight"], s["out"], EPS, residual=s["residual"], residual_out=s["residual_out"],
                    scales=s["scales"], group=s["group"] if s["case"]["out"] not in ("row", "bf16") else 0)
        return dict(out=s["out"], residual=s["residual_out"], scales=s["scales"])
    if s["kind"] == "prefill":
        mp.linear_prefill(s["q"], s["k"], s["v"], s["g"], s["cu"], s["states"], s["src"], s["dst"], s["out"], max(s["lens"]),
                          workspace=s["workspace"])
    else:
        mp.linear_decode(s["q"], s["k"], s["v"], s["g"], s["states"], s["src"], s["dst"], s["out"], q_tokens=s["case"]["rows"])
    return dict(out=s["out"], states=s["states"])


# ---------------------------------------------------------------------------- the plain forms
def _plain_linear(s):
    """In chunks of up to 128 tokens; every chunk's start from the decayed sums of all chunks before it."""
    case, h, lens = s["case"], s["case"]["h_kv"], s["lens"]
    b, grp = len(lens), case["h_q"] // case["h_kv"]
    c = min(128, max(lens))
    nc = -(-max(lens) // c)
    i = torch.arange(nc * c, device=DEV)
    at = (s["cu"][:-1, None] + i).clamp(max=s["k"].shape[0] - 1).long()                        # [B, nc c]
    inside = i < torch.diff(s["cu"])[:, None]
    heads = lambda x: torch.where(inside[..., None, None], x[at].float(), 0.0).transpose(1, 2)  # noqa: E731
    k, v = heads(s["k"]).reshape(b, h, nc, c, D), heads(s["v"]).reshape(b, h, nc, c, D)
    q = heads(s["q"]).reshape(b, h, grp, nc, c, D)
    g = s["g"].double().expand(s["k"].shape[0], h)
    g = torch.where(inside[..., None], g[at], 0.0).transpose(1, 2).reshape(b, h, nc, c).cumsum(-1)   # inclusive, in 64 bits
    total = g[..., -1].cumsum(-1)                                                              # [B, h, nc]
    tail = torch.exp(g[..., -1:] - g).float()
    sums = torch.matmul((k * tail[..., None]).transpose(-1, -2), v).reshape(b, h, nc, D * D)
    # start n: everything of the chunks r < n, decayed from the end of r to the end of n - 1
    ends = torch.nn.functional.pad(total, (1, 0))                                              # [B, h, nc + 1]
    before = torch.arange(nc, device=DEV) < torch.arange(nc + 1, device=DEV)[:, None]
    weight = torch.exp(torch.where(before, ends[..., :, None] - total[..., None, :], -math.inf)).float()
    src = s["src"].long()
    first = torch.where((src >= 0)[:, None, None, None], s["states"][src.clamp(min=0)], 0.0).reshape(b, h, 1, D * D)
    start = (torch.matmul(weight, sums) + torch.exp(ends).float()[..., None] * first).view(b, h, nc + 1, D, D)
    decay = torch.exp(torch.where(torch.ones(c, c, dtype=torch.bool, device=DEV).tril(), g[..., :, None] - g[..., None, :], -math.inf)).float()
    x = torch.matmul(q, k.transpose(-1, -2)[:, :, None]) * decay[:, :, None]
    o = torch.matmul(x, v[:, :, None]) + torch.matmul(q, start[:, :, None, :-1]) * torch.exp(g).float()[:, :, None, ..., None]
    o = (o * SCALE).reshape(b, case["h_q"], nc * c, D).transpose(1, 2)[inside].to(torch.bfloat16)
    s["states"][s["dst"].long()] = start[:, :, -1]
    return dict(out=o, states=s["states"])


def _plain_norm(s):
    x, w = s["x"].float(), s["weight"].float()
    if s["residual"] is not None:
        x = (x + s["residual"].float()).to(torch.bfloat16).float()
    total = x.to(torch.bfloat16) if s["residual"] is not None else None
    rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    y = x * w                                          # exact: eight bits times eight
    if s["scales"] is None:
        return dict(out=(y * rstd).to(torch.bfloat16), residual=total, scales=None)
    n, width = y.shape
    short = -width % s["group"]
    y = torch.nn.functional.pad(y, (0, short)).view(n, -1, s["group"]).double()     # codes next to a border: 64 bits
    top = y.abs().amax(-1, keepdim=True)
    codes = torch.where(top > 0, 448 * y / torch.where(top > 0, top, 1.0), 0.0).float().to(torch.float8_e4m3fn)
    scales = torch.where(top > 0, top.float() * rstd[..., None] / 448, 1.0)[..., 0]
    return dict(out=codes.view(n, -1)[:, :width], residual=total, scales=scales)


def run(state):
    if own:
        return _run_own(state)
    return _plain_norm(state) if state["kind"] == "norm" else _plain_linear(state)


# ---------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["kind"] == "norm":
        n = case["rows"] * case["width"]
        group = case["width"] if case["out"] == "row" else int(case["out"]) if case["out"] != "bf16" else 0
        scales = 4 * case["rows"] * -(-case["width"] // group) if group else 0
        return dict(bytes=n * (2 + (4 if case["residual"] else 0) + (1 if group else 2)) + scales + 2 * case["width"], flops=5 * n)
    lens, h_q, h = _lens(case), case["h_q"], case["h_kv"]
    t, b = sum(lens), len(lens)
    state = b * h * D * D * 4
    return dict(bytes=t * (2 * h_q + 2 * h) * 2 * D + (4 * t * h if case["decay"] == "token" else 4 * h) + state * (2 if case.get("carried", True) else 1),
                flops=t * (h_q + h) * 2 * D * D)


# ---------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if s["kind"] == "norm":
        return _exact_norm(s)
    h, grp = case["h_kv"], case["h_q"] // case["h_kv"]
    states, out = s["states"].double(), torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    src, dst, at = s["src"].tolist(), s["dst"].tolist(), 0
    block = 256
    for b, n in enumerate(s["lens"]):
        now = states[src[b]].clone() if src[b] >= 0 else torch.zeros(h, D, D, dtype=torch.float64, device=DEV)
        for t0 in range(at, at + n, block):
            t1 = min(at + n, t0 + block)
            q, k, v = (s[x][t0:t1].double().transpose(0, 1).contiguous() for x in "qkv")       # [heads, m, D]
            g = s["g"].double().expand(s["k"].shape[0], h)[t0:t1].T                            # [h, m]
            m = t1 - t0
            # decay[i][j]: the product of exp(g) over the tokens j + 1 .. i
            reach = torch.ones(m, m, dtype=torch.float64, device=DEV).tril()
            sums = torch.cumsum(g, -1)
            decay = torch.exp((sums[:, :, None] - sums[:, None, :]).clamp(max=0)) * reach
            old = torch.exp(sums)
            for hk in range(h):
                mine = slice(hk * grp, hk * grp + grp)
                x = (q[mine] @ k[hk].T.contiguous()) * decay[hk]
                out[t0:t1, mine] = ((x @ v[hk] + (q[mine] * old[hk][:, None]) @ now[hk]) * SCALE).transpose(0, 1)
                now[hk] = old[hk, -1] * now[hk] + (k[hk] * decay[hk, -1][:, None]).T.contiguous() @ v[hk]
        states[dst[b]] = now
        at += n
    return dict(out=out, states=states)


def _exact_norm(s):
    x = s["x"].double()
    total = None
    if s["residual"] is not None:
        total = (x + s["residual"].double()).float().to(torch.bfloat16).double()
        x = total
    rstd = 1 / torch.sqrt((x * x).mean(-1) + EPS)
    y = x * s["weight"].double() * rstd[:, None]
    if s["scales"] is None:
        return dict(out=y, residual=total, scales=None)
    codes, scales = torch.empty_like(y), torch.empty(s["scales"].shape, dtype=torch.float64, device=DEV)
    for n, c0 in enumerate(range(0, y.shape[1], s["group"])):
        part = (x * s["weight"].double())[:, c0:c0 + s["group"]]
        top = part.abs().amax(-1)
        scales[:, n] = torch.where(top > 0, top * rstd / 448, 1.0)
        a = torch.where(top[:, None] > 0, 448 * part.abs() / torch.where(top > 0, top, 1.0)[:, None], 0.0)
        bits = a.clamp(min=2.0 ** -6).view(torch.int64)              # its power of two; below 2^-6 that of 2^-6
        step = (bits & (2047 << 52)).view(torch.float64) / 8           # three bits behind the first
        codes[:, c0:c0 + s["group"]] = torch.sign(part) * torch.round(a / step) * step
    return dict(out=codes, residual=total, scales=scales)
