"""Operators for training models beyond the stack's own block, as cases that can be timed and compared.

Four operators, each through the public entry points of paper_2407_00952_amd.binding:

  attention  softmax attention over packed records of any lengths, key/value heads shared by query heads, forward and the
             backward that recomputes the probabilities
  rmsnorm    root-mean-square norm with the residual's addition, result in bf16, in MXFP8 (codes and scales) or both, and
             its backward
  distill    distillation from a teacher's top logits, with the labels' cross-entropy beside it: loss and gradient
  embed      embedding lookup with scaling, and the gradient of the table

Every operator has its plain form here too, in elementary torch operations of 32 bits, and its definition in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-5
BF = torch.bfloat16
F32 = torch.float32


def _attention(name, lens, heads, kv_heads, head, step=True, causal=True, window=0, pad=0):
    return {"name": name, "op": "attention", "lens": ",".join(map(str, lens)), "pad": pad, "heads": heads,
            "kv_heads": kv_heads, "head": head, "step": step, "causal": causal, "window": window}


def _rmsnorm(name, T, d, res, out, step=True, dgamma=True):
    return {"name": name, "op": "rmsnorm", "T": T, "d": d, "res": res, "out": out, "step": step, "dgamma": dgamma}


def _distill(name, T, vocab, ld, dtype, k, tau, kd, ce, step=True):
    return {"name": name, "op": "distill", "T": T, "vocab": vocab, "ld": ld, "dtype": dtype, "k": k, "tau": tau, "kd": kd,
            "ce": ce, "step": step}


def _embed(name, T, vocab, d, dtype, scale, step=True):
    return {"name": name, "op": "embed", "T": T, "vocab": vocab, "d": d, "dtype": dtype, "scale": scale, "step": step}


def listed():
    return [
        # one short record of one client, GPT-2 small: the latency of a forward and a backward pass
        _attention("attention_one_record", [37], 12, 12, 64),
        # a server batch of prompt-completion records as they are, 16 to 512 tokens, packed without padding, GPT-2 medium;
        # one record came empty, and the buffers have room behind the last record
        _attention("attention_records", [16 + (i * 197) % 497 for i in range(63)] + [0], 16, 16, 64, pad=77),
        # a model that shares its key/value heads, heads of 128: few long records and some short ones
        _attention("attention_shared_heads", [4096, 1900, 1, 2777, 3500, 64, 4046], 32, 8, 128),
        # the loss of one long record is wanted, no gradient
        _attention("attention_long_forward", [16384], 16, 16, 64, step=False),
        # a single token on its way through a compressed model
        _rmsnorm("rmsnorm_one_token", 1, 1024, "bf16", "codes", step=False),
        # the headline workload's rows: residual stream in fp32, bf16 for the adapters, codes for the frozen product
        _rmsnorm("rmsnorm_medium", 32768, 1024, "fp32", "both"),
        # a wide model with its residual stream in bf16 and a frozen norm, rows that fill no whole tile
        _rmsnorm("rmsnorm_wide", 10001, 5120, "bf16", "bf16", dgamma=False),
        # one record, a teacher that sends its top 8
        _distill("distill_one_record", 37, 50257, 50257, "bf16", 8, 2.0, 1.0, 0.0),
        # a batch against the whole GPT-2 vocabulary in dense rows, labels beside the teacher
        _distill("distill_batch", 16384, 50257, 50257, "bf16", 64, 2.0, 0.5, 0.5),
        # logits kept in fp32, in padded rows
        _distill("distill_fp32", 2053, 32003, 32064, "fp32", 16, 1.0, 1.0, 0.25),
        # one short record's lookup
        _embed("embed_one_record", 37, 50257, 768, "bf16", 1.0, step=False),
        # a large batch, lookup and the gradient of the whole table
        _embed("embed_batch", 65536, 50257, 1024, "bf16", 32.0),
    ]


def _log(rng, lo, hi):
    return max(1, round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    op = rng.choice(["attention"] * 2 + ["rmsnorm", "distill", "embed"])
    step = rng.random() < 0.75
    if op == "attention":
        most = _log(rng, 1, 16384)
        lens = [rng.randint(0, most) if rng.random() < 0.8 else _log(rng, 1, most) for _ in range(_log(rng, 1, 64))]
        lens.append(most)
        rng.shuffle(lens)
        kv, group = rng.choice([1, 2, 4, 8, 12, 16]), rng.choice([1, 1, 2, 4, 8])
        causal = rng.random() < 0.8
        return _attention("", lens, min(kv * group, 40 // kv * kv), kv, rng.choice([64, 128]), step, causal,
                          _log(rng, 1, most) if causal and rng.random() < 0.3 else 0, rng.choice([0, 0, 5, 130]))
    if op == "rmsnorm":
        out = rng.choice(["bf16", "codes", "both"])
        d = 8 * _log(rng, 8, 1024) if out == "bf16" else 32 * _log(rng, 2, 256)
        return _rmsnorm("", _log(rng, 1, 65536), d, rng.choice(["none", "bf16", "fp32"]), out, step, rng.random() < 0.6)
    if op == "distill":
        vocab = _log(rng, 500, 152064)
        return _distill("", _log(rng, 1, 32768), vocab, vocab + rng.choice([0, 0, 1, 8 - vocab % 8, 64]),
                        rng.choice(["bf16", "fp32"]), min(rng.choice([1, 5, 8, 20, 64, 100]), vocab // 4),
                        rng.choice([1.0, 1.0, 2.0, 4.0, 0.5]), rng.choice([1.0, 0.5]), rng.choice([0.0, 0.5, 1.0]), step)
    return _embed("", _log(rng, 1, 131072), _log(rng, 500, 152064), 8 * _log(rng, 8, 512), rng.choice(["bf16", "fp32"]),
                  rng.choice([1.0, 27.7, 0.125]), step)


def draw(rng):
    ceiling = {}
    for c in listed():
        w = work(c)
        b, f = ceiling.get(c["op"], (0, 0))
        ceiling[c["op"]] = (max(b, w["bytes"]), max(f, w["flops"]))
    while True:
        case = _draw(rng)
        if case["op"] == "attention" and sum(_lens(case)) == 0:
            continue
        w, top = work(case), ceiling[case["op"]]
        if w["bytes"] <= top[0] and w["flops"] <= top[1]:
            del case["name"]
            return case


# ---- inputs -----------------------------------------------------------------------------------------------------
def _lens(case):
    return [int(n) for n in case["lens"].split(",")]


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, std=1.0, mean=0.0, dtype=BF):
    return torch.randn(shape, generator=g, device="cuda", dtype=F32).mul_(std).add_(mean).to(dtype)


def _inputs(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["op"] == "attention":
        H, Hk, D, lens = case["heads"], case["kv_heads"], case["head"], _lens(case)
        T = sum(lens) + case["pad"]
        starts = [0]
        for n in lens:
            starts.append(starts[-1] + n)
        # q | k | v side by side, as one product writes them
        qkv = _normal(g, (T, H + 2 * Hk, D), dtype=F32)
        # the first token of a record draws more attention than the others; the value rows of a head have a common part
        first = torch.tensor([a for a, n in zip(starts, lens) if n > 0], device="cuda")
        qkv[first, H:H + Hk] *= 1.5
        qkv[:, H + Hk:] += 0.5 * torch.randn((1, Hk, D), generator=g, device="cuda")
        s["qkv"] = qkv.to(BF).reshape(T, (H + 2 * Hk) * D)
        s["start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        s["scale"] = D ** -0.5
        s["dout"] = _normal(g, (T, H * D)) if case["step"] else None
    elif case["op"] == "rmsnorm":
        T, d = case["T"], case["d"]
        x = _normal(g, (T, d), dtype=F32)
        # the channel outliers of transformer activations
        cols = torch.randperm(d, generator=g, device="cuda")[:max(d // 128, 1)]
        x[:, cols] *= 8 + 22 * torch.rand(len(cols), generator=g, device="cuda")
        s["x"] = x.to(BF)
        rt = {"none": None, "bf16": BF, "fp32": F32}[case["res"]]
        s["res"] = None if rt is None else _normal(g, (T, d), 2.0, dtype=rt)
        s["gamma"] = _normal(g, (d,), 0.1, 1.0)
        if case["step"]:
            s["du"] = _normal(g, (T, d), 1.0 / T)
            s["dres"] = None if rt is None else _normal(g, (T, d), 1.0 / T, dtype=rt)
    elif case["op"] == "distill":
        T, V, k = case["T"], case["vocab"], case["k"]
        z = torch.empty((T, case["ld"]), dtype=F32, device="cuda").normal_(0.0, 2.0, generator=g)
        # distinct ids of a row: steps of its own through the vocabulary
        a = torch.randint(0, V, (T, 1), generator=g, device="cuda")
        b = torch.randint(1, max(V // k, 2), (T, 1), generator=g, device="cuda")
        ids = (a + b * torch.arange(k, device="cuda")) % V
        gaps = -torch.log(torch.rand((T, k), generator=g, device="cuda").clamp_min(1e-6))
        top = 14.0 - 0.5 * torch.cumsum(gaps, 1)
        # the student has learnt part of it
        z.scatter_add_(1, ids, 0.5 * top)
        s["logits"] = z.to(BF) if case["dtype"] == "bf16" else z
        # some rows of the teacher hold fewer entries, some none
        n = torch.where(torch.rand((T, 1), generator=g, device="cuda") < 0.1,
                        torch.randint(0, k + 1, (T, 1), generator=g, device="cuda"), k)
        ids = torch.where(torch.arange(k, device="cuda") < n, ids, -1)
        right = torch.rand(T, generator=g, device="cuda") < 0.7
        labels = torch.where(right, ids[:, 0], torch.randint(0, V, (T,), generator=g, device="cuda"))
        # a prompt's tokens carry no loss
        w = (torch.rand(T, generator=g, device="cuda") < 0.75).to(F32)
        w[0] = 1.0
        s["ids"], s["top"], s["labels"] = ids.to(torch.int32).contiguous(), top, labels.to(torch.int32)
        s["w"] = w / w.sum()
    else:
        T, V, d = case["T"], case["vocab"], case["d"]
        dt = BF if case["dtype"] == "bf16" else F32
        s["table"] = _normal(g, (V, d), 0.02, dtype=dt)
        # words are as frequent as the inverse of their rank; one token in fifty is padding
        u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
        tok = (torch.exp(u * math.log(V)) - 1).long().clamp_(0, V - 1)
        tok = torch.randperm(V, generator=g, device="cuda")[tok]
        s["tokens"] = torch.where(torch.rand(T, generator=g, device="cuda") < 0.02, -1, tok).to(torch.int32)
        s["dout"] = _normal(g, (T, d), 1.0 / T, dtype=dt) if case["step"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    from paper_2407_00952_amd import binding as B

    def new(shape, dtype):
        return torch.zeros(shape, dtype=dtype, device="cuda")

    def work_space(n):
        s["nws"], s["ws"] = n, torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")

    if case["op"] == "attention":
        H, Hk, D = case["heads"], case["kv_heads"], case["head"]
        T = s["qkv"].shape[0]
        s["o"], s["lse"] = new((T, H * D), BF), new((H, T), F32)
        if case["step"]:
            s["o_lo"], s["dqkv"] = new((T, H * D), BF), torch.zeros_like(s["qkv"])
            work_space(B.slora_attention_bwd_ws_bytes(T, H, Hk, D))
    elif case["op"] == "rmsnorm":
        T, d = s["x"].shape
        if s["res"] is not None:
            s["h"] = torch.empty_like(s["res"])
        if case["out"] != "codes":
            s["u"] = new((T, d), BF)
        if case["out"] != "bf16":
            s["codes"], s["scales"] = new((T, d), torch.uint8), new((T, d // 32), torch.uint8)
            s["values"] = new((T, d), BF)
        if case["step"]:
            s["rho"], s["dh"] = new((T,), F32), torch.empty_like(s["x"] if s["res"] is None else s["res"])
            s["dgamma"] = new((d,), F32) if case["dgamma"] else None
            work_space(B.slora_rmsnorm_bwd_ws_bytes(T, d))
    elif case["op"] == "distill":
        s["loss_tok"], s["loss"] = new((case["T"],), F32), new((1,), F32)
        s["dlogits"] = new((case["T"], case["vocab"]), s["logits"].dtype) if case["step"] else None
    else:
        T, V, d = case["T"], case["vocab"], case["d"]
        s["out"] = new((T, d), s["table"].dtype)
        if case["step"]:
            s["dtable"] = new((V, d), F32)
            work_space(B.slora_embed_bwd_ws_bytes(T, V, d))
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    return (_OWN if own else _PLAIN)[case["op"]](s, case)


def _own_attention(s, c):
    from paper_2407_00952_amd import binding as B
    H, Hk, D, T = c["heads"], c["kv_heads"], c["head"], s["qkv"].shape[0]
    ld = (H + 2 * Hk) * D

    def split(t):
        return t, t[:, H * D:], t[:, (H + Hk) * D:]

    q, k, v = split(s["qkv"])
    n = s["start"].numel() - 1
    head = (n, T, H, Hk, D, s["scale"], c["causal"], c["window"], q, ld, k, ld, v, ld, s["start"])
    B.slora_attention_fwd(*head, s["o"], s.get("o_lo"), H * D, s["lse"])
    if not c["step"]:
        return {"o": s["o"], "lse": s["lse"]}
    dq, dk, dv = split(s["dqkv"])
    B.slora_attention_bwd(*head, s["o"], s["o_lo"], H * D, s["lse"], s["dout"], H * D, dq, ld, dk, ld, dv, ld, s["ws"],
                          s["nws"])
    return {"o": s["o"], "lse": s["lse"], "dqkv": s["dqkv"]}


def _own_rmsnorm(s, c):
    from paper_2407_00952_amd import binding as B
    T, d = c["T"], c["d"]
    rt = B.DTYPE_F32 if c["res"] == "fp32" else B.DTYPE_BF16
    B.slora_rmsnorm_fwd(T, d, rt, s["x"], d, s["res"], s["gamma"], EPS, s.get("h"), s.get("u"), d, s.get("codes"),
                        s.get("scales"), s.get("rho"))
    out = {n: s[n] for n in ("h", "u") if n in s}
    if "codes" in s:
        B.slora_mx_dequantize(T, d, s["codes"], s["scales"], s["values"], d)
        out["values"] = s["values"]
    if c["step"]:
        B.slora_rmsnorm_bwd(T, d, rt, s["du"], d, s.get("h", s["x"]), s["rho"], s["gamma"], s["dres"], s["dh"], None, 0,
                            s["dgamma"], s["ws"], s["nws"])
        out["dh"] = s["dh"]
        if c["dgamma"]:
            out["dgamma"] = s["dgamma"]
    return out


def _own_distill(s, c):
    from paper_2407_00952_amd import binding as B
    dt = B.DTYPE_F32 if c["dtype"] == "fp32" else B.DTYPE_BF16
    B.slora_distill_loss(c["T"], c["vocab"], dt, s["logits"], c["ld"], c["k"], s["ids"], s["top"], c["tau"], c["kd"],
                         s["labels"] if c["ce"] else None, c["ce"], s["w"], s["loss_tok"], s["loss"], s["dlogits"],
                         c["vocab"])
    out = {"loss_tok": s["loss_tok"], "loss": s["loss"]}
    if c["step"]:
        out["dlogits"] = s["dlogits"]
    return out


def _own_embed(s, c):
    from paper_2407_00952_amd import binding as B
    T, V, d = c["T"], c["vocab"], c["d"]
    dt = B.DTYPE_F32 if c["dtype"] == "fp32" else B.DTYPE_BF16
    B.slora_embed_fwd(T, V, d, dt, s["tokens"], s["table"], c["scale"], s["out"], d)
    if not c["step"]:
        return {"out": s["out"]}
    B.slora_embed_bwd(T, V, d, dt, s["tokens"], s["dout"], d, c["scale"], 0, s["dtable"], s["ws"], s["nws"])
    return {"out": s["out"], "dtable": s["dtable"]}


_OWN = {"attention": _own_attention, "rmsnorm": _own_rmsnorm, "distill": _own_distill, "embed": _own_embed}


def _visible(n, c, device):
    """[n, n] truth values: which keys (columns) a query (row) sees, None for all of them"""
    if not c["causal"]:
        return None
    i = torch.arange(n, device=device)
    see = i[None, :] <= i[:, None]
    if c["window"]:
        see &= i[:, None] - i[None, :] < c["window"]
    return see


def _plain_attention(s, c):
    H, Hk, D, T = c["heads"], c["kv_heads"], c["head"], s["qkv"].shape[0]
    qkv = s["qkv"].view(T, H + 2 * Hk, D)
    o, lse = torch.zeros((T, H, D), dtype=BF, device="cuda"), torch.zeros((H, T), dtype=F32, device="cuda")
    dqkv = torch.zeros_like(qkv) if c["step"] else None
    at = 0
    for n in _lens(c):
        if n == 0:
            continue
        see = _visible(n, c, qkv.device)
        # whole groups of query heads that share a key/value head, as many as fit a gigabyte of scores
        per = max(1, min(Hk, (1 << 28) // (n * n) // (H // Hk)))
        for k0 in range(0, Hk, per):
            kh = min(per, Hk - k0)
            G = H // Hk
            q = qkv[at:at + n, k0 * G:(k0 + kh) * G].float().transpose(0, 1).contiguous().view(kh, G, n, D)
            k = qkv[at:at + n, H + k0:H + k0 + kh].float().transpose(0, 1).contiguous()
            v = qkv[at:at + n, H + Hk + k0:H + Hk + k0 + kh].float().transpose(0, 1).contiguous()
            p = torch.matmul(q.view(kh, G * n, D), k.transpose(1, 2).contiguous()).view(kh, G, n, n)
            p.mul_(s["scale"])
            if see is not None:
                p.masked_fill_(~see, -math.inf)
            m = p.amax(-1, keepdim=True)
            p.sub_(m).exp_()
            sums = p.sum(-1, keepdim=True)
            lse[k0 * G:(k0 + kh) * G, at:at + n] = (m + sums.log()).view(kh * G, n)
            p.div_(sums)
            out = torch.matmul(p.view(kh, G * n, n), v)
            o[at:at + n, k0 * G:(k0 + kh) * G] = out.view(kh * G, n, D).transpose(0, 1).to(BF)
            if c["step"]:
                do = s["dout"].view(T, H, D)[at:at + n, k0 * G:(k0 + kh) * G].float().transpose(0, 1).contiguous()
                do = do.view(kh, G * n, D)
                dv = torch.matmul(p.view(kh, G * n, n).transpose(1, 2), do)
                delta = (do * out).sum(-1).view(kh, G, n, 1)
                ds = torch.matmul(do, v.transpose(1, 2).contiguous()).view(kh, G, n, n)
                ds.sub_(delta).mul_(p).mul_(s["scale"])
                ds = ds.view(kh, G * n, n)
                dq = torch.matmul(ds, k)
                dk = torch.matmul(ds.transpose(1, 2), q.view(kh, G * n, D))
                dqkv[at:at + n, k0 * G:(k0 + kh) * G] = dq.view(kh * G, n, D).transpose(0, 1).to(BF)
                dqkv[at:at + n, H + k0:H + k0 + kh] = dk.transpose(0, 1).to(BF)
                dqkv[at:at + n, H + Hk + k0:H + Hk + k0 + kh] = dv.transpose(0, 1).to(BF)
        at += n
    out = {"o": o.view(T, H * D), "lse": lse}
    if c["step"]:
        out["dqkv"] = dqkv.view(T, -1)
    return out


def _plain_mx(u):
    """the values that MXFP8 keeps of bf16 values: blocks of 32, scale 2^(exponent of the largest - 8), 4 significant bits"""
    b = u.float().view(u.shape[0], -1, 32)
    top = b.abs().amax(-1, keepdim=True)
    scale = torch.ldexp(torch.ones_like(top), torch.frexp(top)[1] - 9)
    scale = torch.where(top > 0, scale, 1.0)
    y = b / scale
    step = torch.ldexp(torch.ones_like(y), torch.frexp(y)[1].clamp_min(-5) - 4)
    return ((y / step).round_().mul_(step).clamp_(-448.0, 448.0) * scale).view(u.shape).to(BF)


def _plain_rmsnorm(s, c):
    d = c["d"]
    h = s["x"].float()
    out = {}
    if s["res"] is not None:
        h = h + s["res"].float()
        out["h"] = h.to(s["res"].dtype)
    gamma = s["gamma"].float()
    rho = torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)
    u = (h * rho * gamma).to(BF)
    if c["out"] != "codes":
        out["u"] = u
    if c["out"] != "bf16":
        out["values"] = _plain_mx(u)
    if c["step"]:
        # the backward reads the sum as the forward stored it, and the forward's rho
        h = out["h"].float() if s["res"] is not None else h
        g, xh = s["du"].float(), h * rho
        gg = g * gamma
        dh = rho * (gg - xh * (gg * xh).mean(-1, keepdim=True))
        if s["dres"] is not None:
            dh = dh + s["dres"].float()
        out["dh"] = dh.to(s["x"].dtype if s["res"] is None else s["res"].dtype)
        if c["dgamma"]:
            out["dgamma"] = (g * xh).sum(0)
    return out


def _plain_distill(s, c):
    V, tau = c["vocab"], c["tau"]
    z = s["logits"][:, :V].float()
    ids, on = s["ids"].long(), s["w"] != 0
    valid = (ids >= 0) & (ids < V)
    ids = ids.clamp(0, V - 1)
    has = valid.any(-1) & on
    t = (s["top"] / tau).masked_fill(~valid, -math.inf)
    tm = t.amax(-1, keepdim=True)
    tm = torch.where(tm > -math.inf, tm, 0.0)
    e = (t - tm).exp()
    ts = e.sum(-1, keepdim=True).clamp_min(1e-30)
    p = e / ts
    zt = z / tau
    m = zt.amax(-1, keepdim=True)
    lse = m + (zt - m).exp().sum(-1, keepdim=True).log()
    at = torch.where(p > 0, p * ((t - tm - ts.log()) - (zt.gather(1, ids) - lse)), 0.0)
    loss_tok = torch.where(has, c["kd"] * tau * tau * at.sum(-1), 0.0)
    labels = s["labels"].long()
    lab = on & (labels >= 0) & (labels < V)
    if c["ce"]:
        m1 = z.amax(-1, keepdim=True)
        lse1 = m1 + (z - m1).exp().sum(-1, keepdim=True).log()
        picked = z.gather(1, labels.clamp(0, V - 1)[:, None])
        loss_tok = loss_tok + torch.where(lab, c["ce"] * (lse1 - picked)[:, 0], 0.0)
    out = {"loss_tok": loss_tok, "loss": (loss_tok.double() * s["w"].double()).sum().float().view(1)}
    if c["step"]:
        wk = (c["kd"] * tau * s["w"] * has)[:, None]
        dz = (zt - lse).exp_().mul_(wk)
        dz.scatter_add_(1, ids, -(wk * p))
        if c["ce"]:
            wc = (c["ce"] * s["w"] * lab)[:, None]
            dz.add_((z - lse1).exp_().mul_(wc))
            dz.scatter_add_(1, labels.clamp(0, V - 1)[:, None], -wc)
        out["dlogits"] = dz.to(s["logits"].dtype)
    return out


def _plain_embed(s, c):
    tok = s["tokens"].long()
    ok = (tok >= 0) & (tok < c["vocab"])
    rows = s["table"][tok.clamp(0, c["vocab"] - 1)].float() * c["scale"]
    out = {"out": rows.masked_fill_(~ok[:, None], 0.0).to(s["table"].dtype)}
    if c["step"]:
        dtable = torch.zeros((c["vocab"], c["d"]), dtype=F32, device="cuda")
        dtable.index_add_(0, tok[ok], s["dout"][ok].float())
        out["dtable"] = dtable.mul_(c["scale"])
    return out


_PLAIN = {"attention": _plain_attention, "rmsnorm": _plain_rmsnorm, "distill": _plain_distill, "embed": _plain_embed}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    return {"attention": _exact_attention, "rmsnorm": _exact_rmsnorm, "distill": _exact_distill,
            "embed": _exact_embed}[case["op"]](s, case)


def _exact_attention(s, c):
    H, Hk, D, T = c["heads"], c["kv_heads"], c["head"], s["qkv"].shape[0]
    qkv = s["qkv"].view(T, H + 2 * Hk, D)
    o = torch.zeros((T, H, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((H, T), dtype=torch.float64, device="cuda")
    grad = torch.zeros((T, H + 2 * Hk, D), dtype=torch.float64, device="cuda") if c["step"] else None
    at = 0
    for n in _lens(c):
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        see = _visible(n, c, qkv.device)
        for h in range(H):
            kv = h * Hk // H
            part = [qkv[rows, j].double().requires_grad_(c["step"]) for j in (h, H + kv, H + Hk + kv)]
            score = part[0] @ part[1].T * s["scale"]
            if see is not None:
                score = score.masked_fill(~see, -math.inf)
            l = torch.logsumexp(score, -1)
            y = (score - l[:, None]).exp() @ part[2]
            o[rows, h], lse[h, rows] = y.detach(), l.detach()
            if c["step"]:
                y.backward(s["dout"].view(T, H, D)[rows, h].double())
                for j, t in zip((h, H + kv, H + Hk + kv), part):
                    grad[rows, j] += t.grad
    out = {"o": o.view(T, H * D), "lse": lse}
    if c["step"]:
        out["dqkv"] = grad.view(T, -1)
    return out


def _exact_rmsnorm(s, c):
    T, d = s["x"].shape
    h = s["x"].double()
    out = {}
    if s["res"] is not None:
        h = h + s["res"].double()
        out["h"] = h.clone()
    rms = (h.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt()
    u = h / rms * s["gamma"].double()
    if c["out"] != "codes":
        out["u"] = u
    if c["out"] != "bf16":
        # MXFP8 of the bf16 tensor
        b = u.to(BF).double().view(T, d // 32, 32)
        top = b.abs().amax(-1, keepdim=True)
        scale = torch.where(top > 0, 2.0 ** (torch.floor(torch.log2(top.clamp_min(1e-300))) - 8), 1.0)
        y = (b / scale).clamp(-448, 448).float().to(torch.float8_e4m3fn).double()
        out["values"] = (y * scale).view(T, d)
    if c["step"]:
        if s["res"] is not None:
            h = h.to(s["res"].dtype).double()
        gamma, du = s["gamma"].double(), s["du"].double()
        # rho is a function of the sum that the forward formed, h of what it stored
        dh = (du * gamma) / rms - h * (du * gamma * h).sum(-1, keepdim=True) / (d * rms.pow(3))
        out["dh"] = dh if s["dres"] is None else dh + s["dres"].double()
        if c["dgamma"]:
            out["dgamma"] = (du * h / rms).sum(0)
    return out


def _exact_distill(s, c):
    T, V, tau = c["T"], c["vocab"], c["tau"]
    loss_tok = torch.zeros(T, dtype=torch.float64, device="cuda")
    dlogits = torch.zeros((T, V), dtype=torch.float64, device="cuda") if c["step"] else None
    per = max(1, (1 << 28) // V)
    for r in range(0, T, per):
        rows = slice(r, min(T, r + per))
        z = s["logits"][rows, :V].double()
        ids, labels, w = s["ids"][rows].long(), s["labels"][rows].long(), s["w"][rows].double()
        ok = (ids >= 0) & (ids < V) & (w != 0)[:, None]
        e = torch.where(ok, (s["top"][rows].double() / tau - 14.0 / tau).exp(), 0.0)
        p = e / e.sum(-1, keepdim=True).clamp_min(1e-300)
        at = ids.clamp(0, V - 1)
        lq = torch.log_softmax(z / tau, -1)
        terms = p * (p.clamp_min(1e-300).log() - lq.gather(1, at))
        loss_tok[rows] = c["kd"] * tau ** 2 * terms.sum(-1)
        any_ok = ok.any(-1).double()
        lab = ((w != 0) & (labels >= 0) & (labels < V)).double()
        if c["ce"]:
            l1 = torch.log_softmax(z, -1)
            loss_tok[rows] -= c["ce"] * lab * l1.gather(1, labels.clamp(0, V - 1)[:, None])[:, 0]
        if c["step"]:
            target = torch.zeros_like(z).scatter_add_(1, at, p)
            d = c["kd"] * tau * (lq.exp() * any_ok[:, None] - target)
            if c["ce"]:
                hot = torch.zeros_like(z).scatter_add_(1, labels.clamp(0, V - 1)[:, None], lab[:, None])
                d += c["ce"] * (l1.exp() * lab[:, None] - hot)
            dlogits[rows] = d * w[:, None]
    out = {"loss_tok": loss_tok, "loss": (loss_tok * s["w"].double()).sum().view(1)}
    if c["step"]:
        out["dlogits"] = dlogits
    return out


def _exact_embed(s, c):
    V, d, T = c["vocab"], c["d"], c["T"]
    tok = torch.where((s["tokens"] >= 0) & (s["tokens"] < V), s["tokens"], V).long()      # row V: tokens without a row
    table = torch.cat([s["table"].double() * c["scale"], torch.zeros((1, d), dtype=torch.float64, device="cuda")])
    out = {"out": table.index_select(0, tok)}
    if c["step"]:
        grad = torch.zeros((V + 1, d), dtype=torch.float64, device="cuda")
        grad.scatter_add_(0, tok[:, None].expand(T, d), s["dout"].double() * c["scale"])
        out["dtable"] = grad[:V]
    return out


# ---- what a pass cannot do without ------------------------------------------------------------------------------
def _pairs(n, c):
    """visible (query, key) pairs of a record of n tokens"""
    if not c["causal"]:
        return n * n
    w = c["window"]
    return n * (n + 1) // 2 if not w or w >= n else w * (w + 1) // 2 + (n - w) * w


def work(case):
    op, step = case["op"], case["step"]
    if op == "attention":
        H, Hk, D = case["heads"], case["kv_heads"], case["head"]
        lens = _lens(case)
        T = sum(lens)
        pairs = sum(_pairs(n, case) for n in lens)
        byt = 2 * T * D * (2 * H + 2 * Hk) + 4 * T * H + 4 * (len(lens) + 1)
        if step:
            byt += 2 * T * D * (2 * H + 2 * Hk)
        return {"bytes": byt, "flops": (14 if step else 4) * D * H * pairs}
    if op == "rmsnorm":
        T, d = case["T"], case["d"]
        e = {"none": 0, "bf16": 2, "fp32": 4}[case["res"]]
        n = 2 + 2 * e + {"bf16": 2, "codes": 1.03125, "both": 3.03125}[case["out"]]
        byt = T * d * n + 2 * d
        if step:
            byt += T * d * (2 + (2 * e if e else 2)) + (4 * d if case["dgamma"] else 0)
        return {"bytes": byt, "flops": T * d * (14 if step else 5)}
    if op == "distill":
        T, V, k = case["T"], case["vocab"], case["k"]
        e = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": T * (V * e * (2 if step else 1) + 8 * k + 12) + 4, "flops": T * V * (8 if step else 4)}
    T, V, d = case["T"], case["vocab"], case["d"]
    e = 2 if case["dtype"] == "bf16" else 4
    byt = 4 * T + e * d * (T + min(T, V))
    if step:
        byt += e * T * d + 4 * V * d
    return {"bytes": byt, "flops": T * d * (3 if step else 1)}
