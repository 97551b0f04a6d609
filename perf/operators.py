"""Performance cases of the attention to states that are not the sequence's own: an
encoder's states of another length, a memory that the whole batch shares, and a long
prefix that the whole batch shares.

Kinds:
  train    cross attention of a decoder layer in training: forward and backward;
  forward  its forward alone (evaluation, or the prompt of a generation);
  decode   its forward for one new token of every sequence;
  prefix   serving: the newest T tokens of every sequence over a prefix that is stored
           once for the batch and over the sequence's own rows behind it;
  memory   a sparse self-attention layer whose queries also read M rows shared by the
           batch: the dense part and its join with the sparse part's output.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _case(name, kind, dtype, B, H, H_kv, T, S, D, P=0, ragged=False, views=False):
    """S: rows of the states (prefix: rows a sequence's own buffer holds); P: rows of the
    prefix; ragged: the sequences' states have lengths of their own; views: q and the
    states left where projections wrote them ([B,T,H,D] and [B,S,2,H_kv,D])."""
    return {"name": name, "kind": kind, "dtype": dtype, "B": B, "H": H, "H_kv": H_kv, "T": T, "S": S, "D": D,
            "P": P, "ragged": ragged, "views": views}


def listed():
    return [
        # one token of one sequence over a short sentence: the latency of a call
        _case("decode_S128", "decode", "bf16", 1, 8, 8, 1, 128, 64),
        # generation for a batch of long documents, grouped heads, ragged lengths, states
        # left in the fused projection's output
        _case("decode_S4096", "decode", "bf16", 32, 16, 4, 1, 4096, 128, ragged=True, views=True),
        # the same step of a float32 model, 1500 encoder frames
        _case("decode_fp32_S1500", "decode", "fp32", 4, 8, 8, 1, 1500, 64),
        # training at the shape of this repository's 60M layer, source and target alike long
        _case("train_T1024", "train", "bf16", 8, 8, 8, 1024, 1024, 64),
        # training of a larger head size, grouped heads, padded sources of odd length, views
        _case("train_d128_S2500", "train", "bf16", 2, 16, 4, 1000, 2500, 128, ragged=True, views=True),
        # small heads, a source shorter than the target
        _case("train_d32_S300", "train", "bf16", 16, 8, 2, 512, 300, 32, ragged=True),
        # float32 training with odd lengths
        _case("train_fp32_T333", "train", "fp32", 2, 8, 8, 333, 777, 64),
        # evaluation over a long source, the largest product
        _case("forward_S8192", "forward", "bf16", 4, 8, 8, 2048, 8192, 64),
        # samples drawn from one long prompt: each step reads the prompt for all of them
        _case("prefix_P8192", "prefix", "bf16", 64, 16, 4, 1, 512, 128, P=8192, ragged=True),
        # several new tokens a step (a drafted continuation), a system prompt of odd length
        _case("prefix_T4_P2000", "prefix", "bf16", 16, 8, 2, 4, 200, 64, P=2000, ragged=True),
        # a sparse layer of the 60M model with its 8 query heads on 2, and 256 shared rows
        _case("memory_M256", "memory", "bf16", 8, 8, 2, 1024, 256, 64),
        # a float32 layer with a short memory, odd sizes
        _case("memory_fp32_M100", "memory", "fp32", 4, 8, 8, 1000, 100, 32),
    ]


def draw(rng):
    most = [work(c) for c in listed()]
    most = {k: max(w[k] for w in most) for k in ("bytes", "flops")}

    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choice(["train", "train", "train", "forward", "decode", "decode", "prefix", "prefix", "memory"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        D = rng.choice([64, 64, 128, 32])
        H_kv = rng.choice([1, 2, 4, 8])
        H = H_kv * rng.choice([1, 1, 2, 4])
        P = 0
        if kind in ("train", "forward"):
            B, T, S = log_int(1, 16), log_int(16, 2500), log_int(16, 9000)
        elif kind == "decode":
            B, T, S = log_int(1, 64), 1, log_int(16, 9000)
        elif kind == "prefix":
            B, T, S, P = log_int(2, 96), rng.choice([1, 1, 2, 5, 8]), log_int(16, 1200), log_int(64, 16000)
        else:
            B, T, S = log_int(1, 16), log_int(48, 2500), log_int(4, 600)
        c = _case("", kind, dtype, B, H, H_kv, T, S, D, P, rng.random() < 0.5 and kind != "memory",
                  rng.random() < 0.3)
        del c["name"]
        w = work(c)
        if all(w[k] <= most[k] for k in most):
            return c


def _lens(case):
    """Valid rows of each sequence's states (the last T of them the newest tokens of a
    prefix case): all, or spread over the upper half and more of the range."""
    B, S, T = case["B"], case["S"], case["T"]
    if not case["ragged"]:
        return [S] * B
    low = min(T, S) if case["kind"] == "prefix" else 1
    return [max(low, S - (b * 40503 % 65536) * (S - S // 4) // 65536) for b in range(B)]


def work(case):
    B, H, Hkv, T, S, D, P = (case[x] for x in ("B", "H", "H_kv", "T", "S", "D", "P"))
    es = 2 if case["dtype"] == "bf16" else 4
    rows_q = B * H * T
    kind, lens = case["kind"], _lens(case)
    nbytes = es * D * 2 * rows_q + 4 * rows_q  # q, o, lse
    if kind == "memory":
        rows_k, pairs = Hkv * S, rows_q * S
        nbytes += es * D * rows_q + 4 * rows_q  # the sparse part's output and lse
    else:
        rows_k, pairs = Hkv * sum(lens), H * T * sum(lens)
        if kind == "prefix":
            # query t of a sequence reads its own rows up to the one of token t
            pairs = H * sum(max(0, n - T + 1 + t) for n in lens for t in range(T)) + rows_q * P
            rows_k += Hkv * P
    nbytes += 2 * es * D * rows_k
    flops = 4 * D * pairs  # q.k and p.v
    if kind == "train":
        nbytes += es * D * (2 * rows_q + 2 * Hkv * B * S)  # dO, dq; dk, dv (zeros behind the lengths)
        flops += 10 * D * pairs  # q.k again, dO.v, dq, dk, dv
    return {"bytes": nbytes, "flops": flops}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, H, Hkv, T, S, D, P = (case[x] for x in ("B", "H", "H_kv", "T", "S", "D", "P"))
    dt = DTYPES[case["dtype"]]
    kind = case["kind"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(dt)

    s = {"case": case}
    Bk = 1 if kind == "memory" else B
    if case["views"]:
        s["q"] = normal(B, T, H, D).transpose(1, 2)
        kv = normal(Bk, S, 2, Hkv, D)
        s["k"], s["v"] = (kv[:, :, n].transpose(1, 2) for n in range(2))
    else:
        s["q"], s["k"], s["v"] = normal(B, H, T, D), normal(Bk, Hkv, S, D), normal(Bk, Hkv, S, D)
    s["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
    if kind == "train":
        s["dO"] = normal(B, H, T, D)
    if kind == "prefix":
        s["kp"], s["vp"] = normal(1, Hkv, P, D), normal(1, Hkv, P, D)
    if kind == "memory":
        # what the sparse forward leaves: averages of about 19 values, and the logarithm of
        # a sum of about 19 exponentials
        s["o_s"] = (0.35 * torch.randn((B, H, T, D), generator=g, device="cuda")).to(dt)
        s["lse_s"] = 3.4 + 0.3 * torch.randn((B, H, T), generator=g, device="cuda")
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2606_28560_amd import fibattn as F

    kind, q, k, v, lens = s["case"]["kind"], s["q"], s["k"], s["v"], s["lens"]
    if kind == "prefix":
        o, lse = F.fibattn_prefix_forward(q, s["kp"], s["vp"], k, v, lens)
        return {"o": o, "lse": lse}
    o, lse = F.fibattn_cross_forward(q, k, v, lens)
    if kind == "memory":
        o, lse = F.fibattn_join(s["o_s"], s["lse_s"], o, lse)
    if kind != "train":
        return {"o": o, "lse": lse}
    dq, dk, dv = F.fibattn_cross_backward(q, k, v, o, lse, s["dO"], lens)
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _run_plain(s):
    case = s["case"]
    B, H, Hkv, T, S, D, P = (case[x] for x in ("B", "H", "H_kv", "T", "S", "D", "P"))
    kind, G, tau = case["kind"], H // Hkv, 1.0 / math.sqrt(D)
    dt = s["q"].dtype
    # the query heads of one key/value head side by side as rows
    q = s["q"].float().reshape(B, Hkv, G * T, D)
    k, v = s["k"].float(), s["v"].float()
    logits = torch.matmul(q, k.transpose(2, 3).contiguous()) * tau
    limit = s["lens"]
    if kind == "prefix":
        if limit is None:
            limit = torch.full((B,), S, device=q.device, dtype=torch.int32)
        t = torch.arange(T, device=q.device).repeat(G)
        limit = (limit[:, None] - T + 1 + t[None, :])[:, None, :, None]
    elif limit is not None:
        limit = limit[:, None, None, None]
    if limit is not None:
        keep = torch.arange(S, device=q.device) < limit
        logits = torch.where(keep, logits, torch.full_like(logits, -math.inf))
    if kind == "prefix":
        logits = torch.cat([torch.matmul(q, s["kp"].float().transpose(2, 3).contiguous()) * tau, logits], dim=3)
    top = logits.amax(dim=3, keepdim=True)
    p = torch.exp(logits - top)
    total = p.sum(dim=3, keepdim=True)
    p = p / total
    lse = (top + torch.log(total)).reshape(B, H, T)
    if kind == "prefix":
        o = torch.matmul(p[..., :P], s["vp"].float()) + torch.matmul(p[..., P:].contiguous(), v)
    else:
        o = torch.matmul(p, v)
    if kind == "memory":
        both = torch.logaddexp(lse, s["lse_s"])
        o = (o.reshape(B, H, T, D) * torch.exp(lse - both)[..., None]
             + s["o_s"].float() * torch.exp(s["lse_s"] - both)[..., None])
        return {"o": o.to(dt), "lse": both}
    out = {"o": o.reshape(B, H, T, D).to(dt), "lse": lse}
    if kind == "train":
        g = s["dO"].float().reshape(B, Hkv, G * T, D)
        dp = torch.matmul(g, v.transpose(2, 3).contiguous())
        ds = p * (dp - (g * o).sum(dim=3, keepdim=True)) * tau
        out["dq"] = torch.matmul(ds, k).reshape(B, H, T, D).to(dt)
        out["dk"] = torch.matmul(ds.transpose(2, 3), q).to(dt)
        out["dv"] = torch.matmul(p.transpose(2, 3), g).to(dt)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    B, H, Hkv, T, S, D, P = (case[x] for x in ("B", "H", "H_kv", "T", "S", "D", "P"))
    kind, G = case["kind"], H // Hkv
    lens = _lens(case)
    f64 = {"dtype": torch.float64, "device": "cuda"}
    o, lse = torch.zeros((B, H, T, D), **f64), torch.zeros((B, H, T), **f64)
    grads = kind == "train"
    if grads:
        dq, dk, dv = (torch.zeros(sh, **f64) for sh in ((B, H, T, D), (B, Hkv, S, D), (B, Hkv, S, D)))
    for b in range(B):
        n = lens[b]
        for h in range(H):
            j = h // G
            q = s["q"][b, h].double()
            kb = 0 if kind == "memory" else b
            k, v = s["k"][kb, j, :n].double(), s["v"][kb, j, :n].double()
            x = q @ k.T / math.sqrt(D)
            if kind == "prefix":
                row = torch.arange(T, device="cuda")[:, None] + (n - T)  # the tokens' own rows
                x = x.masked_fill(torch.arange(n, device="cuda")[None, :] > row, -math.inf)
                x = torch.cat([x, q @ s["kp"][0, j].double().T / math.sqrt(D)], dim=1)
                v = torch.cat([v, s["vp"][0, j].double()], dim=0)
            z = torch.logsumexp(x, dim=1)
            w = torch.exp(x - z[:, None])
            y = w @ v
            if kind == "memory":
                # softmax over the union: each part weighs with its share of the sum
                zs = s["lse_s"][b, h].double()
                both = torch.logsumexp(torch.stack([z, zs]), dim=0)
                y = y * torch.exp(z - both)[:, None] + s["o_s"][b, h].double() * torch.exp(zs - both)[:, None]
                z = both
            o[b, h], lse[b, h] = y, z
            if grads:
                u = s["dO"][b, h].double()
                e = w * (u @ v.T - (u * y).sum(1)[:, None]) / math.sqrt(D)
                dq[b, h] = e @ k
                dk[b, j, :n] += e.T @ q
                dv[b, j, :n] += w.T @ u
    out = {"o": o, "lse": lse}
    if grads:
        out.update(dq=dq, dk=dk, dv=dv)
    return out
