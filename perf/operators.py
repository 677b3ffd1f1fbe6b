"""What the time of the serving operators beside the compressed cache is measured on: attention of a batch that shares a
compressed prefix, attention that also adds up how much weight every cached token gets, and the eviction that keeps the
heaviest tokens of a cache by that sum.

A case is a dict of plain values.  `kind` says which operator it takes:

  prefix   attend_prefix: `fan` sequences on each of `n_pre` prefixes, each with tokens of its own behind it
  mass     attend_mass: attention over a cache, and the accumulated attention weight of its tokens
  evict    evict: the heaviest `keep` tokens of every sequence, the first and the last ones protected

A place of a cache with weight 0 holds no token: sequences of different lengths share one layout that way.
Inputs are seeded Gaussians with the structure of the repository's synthetic layers: keys and queries share a mean
direction per head, four key channels are outliers, values are plain.
"""
import math

import numpy as np
import torch

own = False

BF16, F32 = "bf16", "f32"


# ---------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one layer (8 KV heads) of a prompt of 16k tokens compressed 4x, four samples drawn from it: the latency of a token
        dict(name="prefix one layer", kind="prefix", dtype=BF16, d=128, n_pre=8, fan=4, g=4, nq=1, count_p=4096, stride_p=4096, count_s=57,
             stride_s=64),
        # all layers of a 32k prompt compressed 4x, sixteen sessions on it, a few hundred own tokens each
        dict(name="prefix sessions", kind="prefix", dtype=BF16, d=128, n_pre=256, fan=16, g=4, nq=1, count_p=8192, stride_p=8192, count_s=301,
             stride_s=512),
        # one layer, 64 sessions on one long prefix, five queries a head (drafted tokens): many queries to a prefix
        dict(name="prefix drafted", kind="prefix", dtype=BF16, d=128, n_pre=8, fan=64, g=4, nq=5, count_p=16385, stride_p=16400, count_s=130,
             stride_s=160),
        # single precision, narrow heads, odd numbers everywhere
        dict(name="prefix single precision", kind="prefix", dtype=F32, d=64, n_pre=3, fan=5, g=2, nq=3, count_p=1000, stride_p=1024, count_s=33,
             stride_s=33),
        # one decode step of one layer, its cache's masses brought forward: the latency of a token, ragged length
        dict(name="mass one layer", kind="mass", dtype=BF16, d=128, n_seq=8, count=4357, stride=4608, g=4, nq=1, visible=4357, decay=1.0),
        # the same for all layers of two concurrent sessions (bandwidth), older weight fading
        dict(name="mass sessions", kind="mass", dtype=BF16, d=128, n_seq=512, count=8321, stride=8448, g=4, nq=1, visible=8321, decay=0.98),
        # the last 64 queries of a prompt judge the prompt, each sees what lies in front of it
        dict(name="mass window", kind="mass", dtype=BF16, d=128, n_seq=8, count=8704, stride=8704, g=4, nq=64, visible=8641, decay=0.0),
        # a whole prompt against itself, causal, one layer
        dict(name="mass prompt", kind="mass", dtype=BF16, d=128, n_seq=8, count=4096, stride=4096, g=4, nq=4096, visible=1, decay=0.0),
        # single precision, narrow heads, the first queries see nothing
        dict(name="mass single precision", kind="mass", dtype=F32, d=64, n_seq=6, count=1501, stride=1504, g=2, nq=37, visible=-4, decay=0.5),
        # one layer's 16k cache brought down to a quarter
        dict(name="evict one layer", kind="evict", dtype=BF16, d=128, n_seq=8, count=16384, stride=16384, keep=4096, sink=4, recent=256),
        # the whole stack of a model at 32k, to a quarter (bandwidth)
        dict(name="evict model", kind="evict", dtype=BF16, d=128, n_seq=256, count=32768, stride=32768, keep=8192, sink=256, recent=256),
        # single precision, narrow heads, a small cache with a budget that is not round
        dict(name="evict single precision", kind="evict", dtype=F32, d=64, n_seq=5, count=1111, stride=1120, keep=301, sink=3, recent=17),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prefix", "prefix", "mass", "mass", "mass", "evict"])
    dtype = rng.choice([BF16, BF16, BF16, F32])
    d = rng.choice([128, 128, 64])
    most = 1 << 20 if dtype == BF16 else 1 << 18          # tokens in all
    if kind == "prefix":
        n_pre = _log_uniform(rng, 1, 128)
        count_p = _log_uniform(rng, 64, min(20000, most // n_pre))
        g, nq = rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 1, 2, 3, 5])
        # queries x tokens of all prefixes, bounded by the largest case of its type
        room = (1 << 27 if dtype == BF16 else 1 << 25) // (n_pre * count_p * g * nq)
        fan = _log_uniform(rng, 1, max(1, min(128, room, 8192 // n_pre)))
        count_s = min(_log_uniform(rng, 1, 600), max(1, most // (n_pre * fan)))
        return dict(kind=kind, dtype=dtype, d=d, n_pre=n_pre, fan=fan, g=g, nq=nq, count_p=count_p, stride_p=count_p + rng.randrange(0, 40),
                    count_s=count_s, stride_s=count_s + rng.randrange(0, 40))
    if kind == "mass":
        g = rng.choice([1, 2, 4, 8])
        form = rng.choice(["token", "token", "window", "prompt"])
        n_seq = _log_uniform(rng, 1, 256 if form == "token" else 16)
        top = min(20000, most // n_seq) if form != "prompt" else 4096
        count = _log_uniform(rng, 16, top)
        pairs = (1 << 28 if dtype == BF16 else 1 << 26) // (n_seq * count * g)
        if form == "token":
            nq, visible = rng.choice([1, 1, 1, 2, 3]), count
        elif form == "window":
            nq = max(1, min(_log_uniform(rng, 2, 128), pairs, count))
            visible = count - nq + 1
        else:
            nq = max(1, min(count, pairs))
            visible = count - nq + 1
        return dict(kind=kind, dtype=dtype, d=d, n_seq=n_seq, count=count, stride=count + rng.randrange(0, 100), g=g, nq=nq, visible=visible,
                    decay=rng.choice([0.0, 0.9, 1.0]))
    n_seq = _log_uniform(rng, 1, 256)
    count = _log_uniform(rng, 64, min(60000, 4 * most // n_seq))
    keep = max(1, int(count * rng.uniform(0.05, 0.9)))
    sink = rng.randrange(0, keep // 4 + 1)
    return dict(kind=kind, dtype=dtype, d=d, n_seq=n_seq, count=count, stride=count + rng.randrange(0, 100), keep=keep, sink=sink,
                recent=rng.randrange(0, (keep - sink) // 2 + 1))


def _types(case):
    return (torch.bfloat16, 2) if case["dtype"] == BF16 else (torch.float32, 4)


def work(case):
    """Keys, values, weights, queries read once, outputs written once; four operations per (query, token, column) of an
    attention, two more where the masses are added up."""
    elem, d = _types(case)[1], case["d"]
    row = 2 * d * elem
    if case["kind"] == "prefix":
        n_seq, n_q = case["fan"] * case["n_pre"], case["g"] * case["nq"]
        tokens = case["n_pre"] * case["count_p"] + n_seq * case["count_s"]
        return {"bytes": tokens * (row + 4) + n_seq * n_q * (row + 4), "flops": 4 * d * n_seq * n_q * (case["count_p"] + case["count_s"])}
    if case["kind"] == "mass":
        n_seq, n_q, count, nq, first = case["n_seq"], case["g"] * case["nq"], case["count"], case["nq"], case["visible"]
        pairs = sum(min(count, max(0, first + i)) for i in range(nq)) * case["g"]
        reads = 12 if case["decay"] else 8
        return {"bytes": n_seq * count * (row + reads) + n_seq * n_q * (row + 4), "flops": 6 * d * n_seq * pairs}
    kept = case["n_seq"] * case["keep"]
    return {"bytes": case["n_seq"] * (case["count"] * 8 + 4) + kept * (2 * row + 12), "flops": case["n_seq"] * case["count"]}


# --------------------------------------------------------------------------------------------------------- the inputs
def _layer(gen, n_seq, n, d, dtype, mean=None, scale=None):
    """Keys and values of n_seq heads: a mean direction of norm 2 and four outlier channels per head."""
    if mean is None:
        mean = torch.randn(n_seq, d, generator=gen, device="cuda")
        mean = 2.0 * mean / mean.norm(dim=1, keepdim=True)
        scale = torch.ones(n_seq, d, device="cuda")
        scale.scatter_(1, torch.rand(n_seq, d, generator=gen, device="cuda").argsort(dim=1)[:, :4], 8.0)
    K = torch.randn(n_seq, n, d, generator=gen, device="cuda").add_(mean[:, None]).mul_(scale[:, None]).to(dtype)
    V = torch.randn(n_seq, n, d, generator=gen, device="cuda").to(dtype)
    return K, V, mean, scale


def _queries(gen, mean, shape, dtype):
    return (torch.randn(*shape, generator=gen, device="cuda") + mean[:, None, None]).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) % (1 << 62) + 17)
    dtype, d = _types(case)[0], case["d"]
    rand = lambda *shape: torch.rand(*shape, generator=gen, device="cuda")
    s = dict(case)
    if case["kind"] == "prefix":
        n_pre, fan, n_seq = case["n_pre"], case["fan"], case["fan"] * case["n_pre"]
        s["K_p"], s["V_p"], mean, scale = _layer(gen, n_pre, case["stride_p"], d, dtype)
        # survivors of two halvings, the last tokens of the prompt as they were
        s["w_p"] = torch.full((n_pre, case["stride_p"]), 4.0, device="cuda")
        s["w_p"][:, case["count_p"] - case["count_p"] // 16:] = 1.0
        mean, scale = mean.repeat(fan, 1), scale.repeat(fan, 1)               # sequence s stands on prefix s mod n_pre
        s["K_s"], s["V_s"], _, _ = _layer(gen, n_seq, case["stride_s"], d, dtype, mean, scale)
        length = 1 + (rand(n_seq, 1) * case["count_s"]).long().clamp_(max=case["count_s"] - 1)
        s["w_s"] = (torch.arange(case["stride_s"], device="cuda")[None] < length).float()
        s["Q"] = _queries(gen, mean, (n_seq, case["g"], case["nq"], d), dtype)
    elif case["kind"] == "mass":
        n_seq = case["n_seq"]
        s["K"], s["V"], mean, _ = _layer(gen, n_seq, case["stride"], d, dtype)
        # a compressed cache with a few places that hold nothing; a prompt against itself is not compressed
        w = torch.exp2(torch.floor(rand(n_seq, case["stride"]) * 3.0)) if case["visible"] >= case["count"] else torch.ones(n_seq, case["stride"], device="cuda")
        s["w"] = w * (rand(n_seq, case["stride"]) < 0.97)
        s["Q"] = _queries(gen, mean, (n_seq, case["g"], case["nq"], d), dtype)
        s["mass"] = rand(n_seq, case["stride"]) * (2.0 * case["g"] * case["nq"] / case["count"])
        s["mass_out"] = s["mass"].clone()
    else:
        n_seq = case["n_seq"]
        s["K"], s["V"], _, _ = _layer(gen, n_seq, case["stride"], d, dtype)
        s["w"] = (rand(n_seq, case["stride"]) < 0.99).float()
        # accumulated weights are heavy-tailed, and tokens that nothing looked at have none
        mass = torch.exp(1.5 * torch.randn(n_seq, case["stride"], generator=gen, device="cuda"))
        s["mass"] = mass * (rand(n_seq, case["stride"]) < 0.9)
    if own:
        import paper_2502_07861_amd as bk
        s["p"] = p = bk.make_params(d, 64, 2, dtype, log_c=0.0)
        if case["kind"] == "prefix":
            need = bk.attend_prefix_workspace_bytes(p, case["n_pre"], case["fan"] * case["n_pre"], case["g"], case["nq"])
        elif case["kind"] == "mass":
            need = bk.attend_mass_workspace_bytes(p, case["n_seq"], case["count"], case["g"], case["nq"])
        else:
            need = bk.evict_workspace_bytes(p, case["n_seq"], case["count"])
        s["workspace"] = torch.empty(need, device="cuda", dtype=torch.uint8)
    return s


# ----------------------------------------------------------------------------------------------------- the plain forms
def _logits(Q, K, w):
    """ln of w_j exp(<k_j, q> / sqrt d) in single precision, -inf where there is no token.  Q [n, queries, d], K [n, tokens, d]."""
    x = torch.matmul(Q.float(), K.float().transpose(1, 2)) / math.sqrt(Q.shape[-1])
    live = (w > 0)[:, None]
    return torch.where(live, x + torch.log(torch.where(w > 0, w, 1.0))[:, None], -math.inf)


def _weights(x):
    """exp(x - its row's largest), the row's sum and ln of the sum of exp(x); rows of nothing give zeros and -inf."""
    top = x.amax(dim=-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    e = torch.exp(x - top)
    total = e.sum(dim=-1, keepdim=True)
    return e, total, (top + torch.log(total)).squeeze(-1)


def _prefix_plain(s):
    n_pre, fan, n_q, d = s["n_pre"], s["fan"], s["g"] * s["nq"], s["d"]
    cp, cs = s["count_p"], s["count_s"]
    K_p, V_p, w_p = s["K_p"][:, :cp], s["V_p"][:, :cp].float(), s["w_p"][:, :cp]
    K_s, V_s, w_s = s["K_s"][:, :cs], s["V_s"][:, :cs].float(), s["w_s"][:, :cs]
    by_prefix = lambda t: t.reshape(fan, n_pre, n_q, -1).transpose(0, 1).reshape(n_pre, fan * n_q, -1)
    by_sequence = lambda t: t.reshape(n_pre, fan, n_q, -1).transpose(0, 1).reshape(fan * n_pre, n_q, -1)
    Q = s["Q"].reshape(fan * n_pre, n_q, d)
    x = torch.cat([by_sequence(_logits(by_prefix(Q), K_p, w_p)), _logits(Q, K_s, w_s)], dim=-1)
    e, total, lse = _weights(x)
    V_p, V_s = torch.where((w_p > 0)[..., None], V_p, 0.0), torch.where((w_s > 0)[..., None], V_s, 0.0)
    z = by_sequence(torch.matmul(by_prefix(e[..., :cp]), V_p)) + torch.matmul(e[..., cp:], V_s)
    z = z / torch.where(total > 0, total, 1.0)
    return z.to(s["Q"].dtype).reshape(s["Q"].shape), lse.reshape(s["Q"].shape[:3])


def _mass_plain(s):
    count, n_q, nq = s["count"], s["g"] * s["nq"], s["nq"]
    w = s["w"][:, :count]
    x = _logits(s["Q"].reshape(s["n_seq"], n_q, s["d"]), s["K"][:, :count], w)
    # query i of a head sees the first visible + i tokens
    sees = s["visible"] + torch.arange(n_q, device="cuda") % nq
    if s["visible"] < count:
        x = torch.where(torch.arange(count, device="cuda") < sees[:, None], x, -math.inf)
    e, total, lse = _weights(x)
    e = e / torch.where(total > 0, total, 1.0)
    z = torch.matmul(e, torch.where((w > 0)[..., None], s["V"][:, :count].float(), 0.0))
    mass = s["mass"].clone()
    mass[:, :count] = s["decay"] * mass[:, :count] + e.sum(dim=1)
    return z.to(s["Q"].dtype).reshape(s["Q"].shape), lse.reshape(s["Q"].shape[:3]), mass


def _evict_plain(s):
    count, keep = s["count"], s["keep"]
    w = s["w"][:, :count]
    place = torch.arange(count, device="cuda")
    window = (place < s["sink"]) | (place >= count - s["recent"])
    # heaviest first, the windows in front of them, places without a token behind; ties go to the lowest place
    rank = torch.where(w > 0, torch.where(window, math.inf, s["mass"][:, :count]), -math.inf)
    pick = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :keep]
    there = torch.gather(w, 1, pick) > 0
    pick = torch.sort(torch.where(there, pick, count), dim=1).values
    there = pick < count
    pick = pick.clamp(max=count - 1)
    rows = pick[..., None].expand(-1, -1, s["d"])
    take = lambda t: torch.where(there, torch.gather(t, 1, pick), 0.0)
    take_rows = lambda t: torch.where(there[..., None], torch.gather(t, 1, rows), 0.0)
    return (take_rows(s["K"]), take_rows(s["V"]), take(s["w"]), take(s["mass"]), torch.where(there, pick, -1).int(),
            there.sum(dim=1).int())


def run(s):
    if own:
        import paper_2502_07861_amd as bk
        if s["kind"] == "prefix":
            return bk.attend_prefix(s["p"], (s["K_p"], s["V_p"], s["w_p"]), (s["K_s"], s["V_s"], s["w_s"]), s["Q"], count_prefix=s["count_p"],
                                    count_own=s["count_s"], workspace=s["workspace"])
        if s["kind"] == "mass":
            return bk.attend_mass(s["p"], s["K"], s["V"], s["w"], s["Q"], s["mass"], count=s["count"], visible=s["visible"], decay=s["decay"],
                                  mass_out=s["mass_out"], workspace=s["workspace"])
        r = bk.evict(s["p"], s["K"], s["V"], s["w"], s["mass"], s["keep"], n_sink=s["sink"], n_recent=s["recent"], count=s["count"],
                     workspace=s["workspace"])
        return r["K"], r["V"], r["w"], r["mass"], r["idx"], r["count"]
    return {"prefix": _prefix_plain, "mass": _mass_plain, "evict": _evict_plain}[s["kind"]](s)


# --------------------------------------------------------------------------------------------------------- in 64 bits
def _softmax64(Q, sets, sees=None):
    """One sequence: Q [queries, d], sets of (K, V, w).  Returns (out, ln of the normaliser, probabilities of all tokens)."""
    K, V, w = (torch.cat([t[k] for t in sets]).double() for k in range(3))
    live = w > 0
    x = Q.double() @ K.T * (1.0 / math.sqrt(Q.shape[-1])) + torch.where(live, w, 1.0).log()
    hidden = ~live[None].expand_as(x)
    if sees is not None:
        hidden = hidden | (torch.arange(K.shape[0], device="cuda")[None] >= sees[:, None])
    x = x.masked_fill(hidden, -math.inf)
    lse = torch.logsumexp(x, dim=1)
    prob = torch.exp(x - lse[:, None].masked_fill(torch.isinf(lse)[:, None], 0.0))
    return prob @ V.masked_fill(~live[:, None], 0.0), lse, prob


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "prefix":
        cp, cs, outs, lses = case["count_p"], case["count_s"], [], []
        for i in range(case["n_pre"] * case["fan"]):
            k = i % case["n_pre"]
            z, lse, _ = _softmax64(s["Q"][i].flatten(0, 1), [(s["K_p"][k, :cp], s["V_p"][k, :cp], s["w_p"][k, :cp]),
                                                            (s["K_s"][i, :cs], s["V_s"][i, :cs], s["w_s"][i, :cs])])
            outs.append(z)
            lses.append(lse)
        return torch.stack(outs).view(s["Q"].shape), torch.stack(lses).view(s["Q"].shape[:3])
    if case["kind"] == "mass":
        count, outs, lses = case["count"], [], []
        mass = s["mass"].double()
        sees = case["visible"] + torch.arange(case["nq"], device="cuda").repeat(case["g"])
        for i in range(case["n_seq"]):
            z, lse, prob = _softmax64(s["Q"][i].flatten(0, 1), [(s["K"][i, :count], s["V"][i, :count], s["w"][i, :count])], sees)
            outs.append(z)
            lses.append(lse)
            mass[i, :count] = mass[i, :count] * float(np.float32(case["decay"])) + prob.sum(dim=0)
        return torch.stack(outs).view(s["Q"].shape), torch.stack(lses).view(s["Q"].shape[:3]), mass
    # the kept places by a sort on the host over (class, mass, place); rows are copies
    count, keep, sink, recent = case["count"], case["keep"], case["sink"], case["recent"]
    w, mass = s["w"][:, :count].cpu().numpy(), s["mass"][:, :count].cpu().numpy()
    place = np.arange(count)
    idx = np.full((case["n_seq"], keep), -1, np.int32)
    for i in range(case["n_seq"]):
        group = np.where(w[i] > 0, np.where((place < sink) | (place >= count - recent), 0, 1), 2)
        order = np.lexsort((place, np.where(group == 1, -mass[i].astype(np.float64), 0.0), group))[:keep]
        kept = np.sort(order[group[order] < 2])
        idx[i, :len(kept)] = kept
    idx = torch.from_numpy(idx).cuda()
    safe, there = idx.clamp(min=0).long(), idx >= 0
    one = lambda t: torch.gather(t, 1, safe).double() * there
    rows = lambda t: torch.gather(t, 1, safe[..., None].expand(-1, -1, case["d"])).double() * there[..., None]
    return rows(s["K"]), rows(s["V"]), one(s["w"]), one(s["mass"]), idx, there.sum(dim=1).int()
