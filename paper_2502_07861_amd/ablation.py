"""Ablation grid of the paper's single-layer study on synthetic data (one GPU).

    python -m paper_2502_07861_amd.ablation [--seeds 10] [--json] [--recipe clustered|iid] [--value-factor | --value-augment | --alg1 | --evict]

For block sizes b in {256, 128, 64} and compression rates 2^-T in {1/2, 1/4, 1/8} (the grid of the runtime /
relative-error tables in "Ablation Studies on Single Layer Attention Approximation", arXiv 2502.07861): the first
and the most recent 256 tokens of every KV sequence are kept, the rows in between go through the halving tree
(`bkv_merge_reduce_protected`), and the estimator of Alg. 1 answers a batch of queries from the kept set.  Reported
per cell: the run time of the compression and the relative error ||z - Attn|| / ||Attn|| per query, mean and standard
deviation over seeds, next to independent uniform sampling of the same number of rows in between (the paper's
comparator).  Next to it the relative error of the softmax normaliser sum_i w_i exp(<k_i,q>/sqrt d), the quantity
that balancing the keys alone controls directly (the denominator instance of Alg. 1).  The estimates come from the
attend kernel; exact attention (Eq. 1) is evaluated in float64 with plain tensor operations, as the yardstick.

The inputs are synthetic stand-ins, one layer of 8 KV heads, 4 query heads each, 64 queries per head; the paper's
tables are on Llama-3.1-8B / TriviaQA activations, so only the shape of the study carries over.  Two recipes:
"clustered" (default; synth.clustered_layer_bf16: keys that repeat -- 32 clusters per head, norms as App. B.5
reports them -- which is what a balancing of exp(<k_i,k_j>/sqrt d) can exploit) and "iid" (synth.gqa_layer_bf16:
independent Gaussians around a common mean, where no subset is better than a random one).
ln c per recipe and block size was bisected once on the CPU oracle (oracle/tuning.py, mean |2p - 1| = 0.25 on the first
four blocks of the first two sequences) so that the walk's decisions depend on the kernel weights.  --value-factor: the walk's weights carry the
value factor <v_i,v_j>/r_value^2 of Alg. 2 line 6 (the numerator instance of Alg. 1 selects the kept set), with its own
ln c per block size found the same way.  --value-augment (clustered recipe): the walk sees the value [v / r_value ; 1], i.e. the
factor (<v_i,v_j>/r_value^2 + 1) / 2: one kept set chosen for numerator and denominator together.  --evict: next to both, eviction by
accumulated attention weight at the same budget: half of the queries judge the tokens (`bkv_attend_mass`), the heaviest stay beside the
windows with their own weights (`bkv_evict`), and all kept sets answer the other half.
"""
from __future__ import annotations

import argparse
import json
import sys

import torch

from . import binding, synth

BLOCKS = (256, 128, 64)
ROUNDS = (1, 2, 3)
N_SINK = N_RECENT = 256
N_MID = 8192
SEED_DATA = 0x250207861006
SEED_CLUSTERED = 0x250207861007
LOG_C = {64: -53.9166, 128: -59.3241, 256: -61.8303}            # recipe "iid"
LOG_C_VALUE = {64: -57.0969, 128: -63.0066, 256: -67.8165}      # ... with the value factor
LOG_C_CLUSTERED = {64: -4.2786, 128: -3.4420, 256: -2.9556}     # recipe "clustered"
LOG_C_CLUSTERED_VALUE = {64: -4.6749, 128: -3.8368, 256: -3.3827}
LOG_C_CLUSTERED_AUGMENT = {64: -4.4572, 128: -3.6253, 256: -3.1501}     # ... with the value [v / r ; 1]


def log_c_for(recipe, block, value_gram=False, value_augment=False):
    if value_augment:
        if recipe != "clustered":
            raise ValueError("ln c for the augmented value is tabulated for the clustered recipe only")
        return LOG_C_CLUSTERED_AUGMENT.get(block, 0.0)
    table = {("iid", False): LOG_C, ("iid", True): LOG_C_VALUE, ("clustered", False): LOG_C_CLUSTERED,
             ("clustered", True): LOG_C_CLUSTERED_VALUE}[(recipe, bool(value_gram))]
    return table.get(block, 0.0)


def make_inputs(device="cuda", n_seq=8, n_mid=N_MID, d=128, g=4, nq=64, recipe="clustered"):
    n = N_SINK + n_mid + N_RECENT
    if recipe == "clustered":
        t = synth.clustered_layer_bf16(n_seq=n_seq, n=n, d=d, g=g, nq=nq, seed=SEED_CLUSTERED, device="cpu")
    else:
        t = synth.gqa_layer_bf16(n_seq=n_seq, n=n, d=d, g=g, nq=nq, seed=SEED_DATA, device="cpu")
    return t["K"].to(device).contiguous(), t["V"].to(device).contiguous(), t["Q"].to(device).contiguous()


def exact_attention_f64(K, V, Q):
    """Eq. 1 in float64: softmax(K q / sqrt d)^T V for every query; returns (out [n_seq,g,nq,d], ln of the normaliser)."""
    Kd, Vd, Qd = K.double(), V.double(), Q.double()
    logits = torch.einsum("sgqd,snd->sgqn", Qd, Kd) / (K.shape[-1] ** 0.5)
    lse = torch.logsumexp(logits, dim=-1)
    return torch.einsum("sgqn,snd->sgqd", torch.exp(logits - lse[..., None]), Vd), lse


def uniform_sample_protected(n_seq, n, n_sink, n_recent, T, seed, device):
    """The comparator: windows kept, a uniformly random 2^-T fraction of the rows in between (without replacement,
    independently per sequence).  Returns (idx [n_seq, count] int64 ascending, w [n_seq, count] fp32)."""
    n_mid = n - n_sink - n_recent
    kept = n_mid >> T
    gen = torch.Generator(device="cpu")
    gen.manual_seed(int(seed))
    rows = []
    for _ in range(n_seq):
        pick = torch.randperm(n_mid, generator=gen)[:kept].sort().values + n_sink
        rows.append(torch.cat([torch.arange(n_sink), pick, torch.arange(n - n_recent, n)]))
    idx = torch.stack(rows).to(device)
    w = torch.ones(n_seq, idx.shape[1], dtype=torch.float32)
    w[:, n_sink:n_sink + kept] = float(2 ** T)
    return idx, w.to(device)


def relative_error(z, exact):
    """Mean over all queries of ||z - Attn|| / ||Attn|| (norms over the head dimension)."""
    z, exact = z.double(), exact.double()
    return float(((z - exact).norm(dim=-1) / exact.norm(dim=-1)).mean())


def _std(t):
    return float(t.std()) if t.numel() > 1 else 0.0


def normaliser_error(lse, lse_exact):
    """Mean over all queries of |D_est / D - 1| for the softmax normaliser D (lse = ln D)."""
    return float((torch.exp(lse.double() - lse_exact.double()) - 1.0).abs().mean())


def run(seeds=10, blocks=BLOCKS, rounds=ROUNDS, n_mid=N_MID, n_seq=8, device="cuda", nq=64, keep_outputs=False,
        value_gram=False, recipe="clustered", value_augment=False):
    """The grid.  value_gram: kernel weights with the value factor of Alg. 2 line 6; value_augment: with the factor of the value [v / r ; 1].  keep_outputs: every cell also carries the tensors of its first counted seed (kept indices, weights,
    both estimates, the uniform comparator's indices) and the result the inputs, for checking against a reference."""
    K, V, Q = make_inputs(device, n_seq=n_seq, n_mid=n_mid, nq=nq, recipe=recipe)
    n, d = K.shape[1], K.shape[2]
    exact, lse_exact = exact_attention_f64(K, V, Q)
    cells = []
    for b in blocks:
        for T in rounds:
            if n_mid % (b << T):
                continue
            err_b, err_u, den_b, den_u, ms = [], [], [], [], []
            for s in range(seeds + 1):                      # run 0 warms up and is not counted
                p = binding.make_params(d, b, T, K.dtype, log_c=log_c_for(recipe, b, value_gram, value_augment),
                                        seed=1000 + s, center=True, value_gram=value_gram, value_augment=value_augment)
                e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                e0.record()
                res = binding.merge_reduce_protected(p, K, V, N_SINK, N_RECENT)
                e1.record()
                z, lse_b = binding.attend_kv(p, res["K"], res["V"], res["w"], Q)
                idx_u, w_u = uniform_sample_protected(n_seq, n, N_SINK, N_RECENT, T, 7000 + s, device)
                gi = idx_u[..., None].expand(-1, -1, d)
                zu, lse_u = binding.attend_kv(p, torch.gather(K, 1, gi), torch.gather(V, 1, gi), w_u, Q)
                torch.cuda.synchronize()
                if s == 0:
                    continue
                if s == 1 and keep_outputs:
                    first = dict(idx=res["idx"], w=res["w"], z=z, lse=lse_b, idx_uniform=idx_u, w_uniform=w_u, z_uniform=zu,
                                 lse_uniform=lse_u, seed=1000 + s)
                ms.append(e0.elapsed_time(e1))
                err_b.append(relative_error(z, exact))
                err_u.append(relative_error(zu, exact))
                den_b.append(normaliser_error(lse_b, lse_exact))
                den_u.append(normaliser_error(lse_u, lse_exact))
            tb, tu, tm = torch.tensor(err_b), torch.tensor(err_u), torch.tensor(ms)
            db, du = torch.tensor(den_b), torch.tensor(den_u)
            cells.append(dict(block=b, rate="1/%d" % (1 << T), rounds=T, kept=int(res["K"].shape[1]),
                              compress_ms=float(tm.mean()), balancekv_rel_err=float(tb.mean()), balancekv_std=_std(tb),
                              uniform_rel_err=float(tu.mean()), uniform_std=_std(tu),
                              balancekv_normaliser_err=float(db.mean()), balancekv_normaliser_std=_std(db),
                              uniform_normaliser_err=float(du.mean()), uniform_normaliser_std=_std(du)))
            if keep_outputs:
                cells[-1]["first"] = first
    return dict(workload="%d KV sequences x (%d + %d + %d) tokens, d=%d, %d x %d queries, bf16, synthetic (recipe %s)%s"
                         % (n_seq, N_SINK, n_mid, N_RECENT, d, Q.shape[1], Q.shape[2], recipe,
                            ", weights with the value factor" if value_gram else ""), seeds=seeds, cells=cells,
                **(dict(K=K, V=V, Q=Q, exact=exact) if keep_outputs else {}))


def heavy_tailed(V, seed=77):
    """Value rows rescaled by 2^U(-3.5, 3.5) per token: norms spread over about eight buckets of Alg. 1 line 5."""
    gen = torch.Generator(device="cpu")
    gen.manual_seed(seed)
    scale = torch.exp2(torch.rand(V.shape[0], V.shape[1], generator=gen) * 7.0 - 3.5).to(V.device)
    return (V.float() * scale[..., None]).to(V.dtype)


def run_alg1(seeds=5, block=128, rounds=ROUNDS, n=8192, n_seq=8, device="cuda", nq=64):
    """Alg. 1 as listed (value-norm buckets with one numerator instance each + the keys-only denominator instance, two
    kept sets) next to the single keys-only set and to uniform sampling, on values with heavy-tailed norms.  Per
    rate: time of building the two sets, time of the two-set output line, relative errors."""
    t = synth.gqa_layer_bf16(n_seq=n_seq, n=n, d=128, g=4, nq=nq, seed=SEED_DATA, device="cpu")
    K, Q = t["K"].to(device).contiguous(), t["Q"].to(device).contiguous()
    V = heavy_tailed(t["V"]).to(device).contiguous()
    d = K.shape[2]
    exact, _ = exact_attention_f64(K, V, Q)
    rows = []
    for T in rounds:
        acc = dict(sets_ms=[], attend_ms=[], alg1=[], single=[], uniform=[], kept_num=[], kept_den=[])
        for s in range(seeds + 1):
            pk = binding.make_params(d, block, T, K.dtype, log_c=LOG_C[block], seed=500 + s, center=True)
            pv = binding.make_params(d, block, T, K.dtype, log_c=LOG_C_VALUE[block], seed=500 + s, center=True)
            ev = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
            ev[0].record()
            num = binding.balancekv_sets(pv, binding.BKV_SET_NUMERATOR, K, V, max_buckets=16, emit_slots=False)
            den = binding.balancekv_sets(pk, binding.BKV_SET_DENOMINATOR, K, V, emit_slots=False)
            ev[1].record()
            z, _ = binding.attend_sets(pk, (num["K"], num["V"], num["w"]), (den["K"], den["w"]), Q)
            ev[2].record()
            one = binding.merge_reduce(pk, K, V)
            z1, _ = binding.attend_kv(pk, one["K"], one["V"], one["w"], Q)
            idx_u, w_u = uniform_sample_protected(n_seq, n, 0, 0, T, 9000 + s, device)
            gi = idx_u[..., None].expand(-1, -1, d)
            zu, _ = binding.attend_kv(pk, torch.gather(K, 1, gi), torch.gather(V, 1, gi), w_u, Q)
            torch.cuda.synchronize()
            if s == 0:
                continue
            acc["sets_ms"].append(ev[0].elapsed_time(ev[1])); acc["attend_ms"].append(ev[1].elapsed_time(ev[2]))
            acc["alg1"].append(relative_error(z, exact)); acc["single"].append(relative_error(z1, exact))
            acc["uniform"].append(relative_error(zu, exact))
            acc["kept_num"].append(float(num["count"].float().mean())); acc["kept_den"].append(float(den["count"].float().mean()))
        m = {k: float(torch.tensor(v).mean()) for k, v in acc.items()}
        m.update({k + "_std": float(torch.tensor(acc[k]).std()) for k in ("alg1", "single", "uniform")})
        m.update(rate="1/%d" % (1 << T), block=block)
        rows.append(m)
    return dict(workload="%d KV sequences x %d tokens, d=%d, 4 x %d queries, bf16, synthetic, value norms x 2^U(-3.5,3.5)"
                         % (n_seq, n, d, nq), seeds=seeds, rows=rows)


def run_evict(seeds=5, block=128, rounds=ROUNDS, n_mid=N_MID, n_seq=8, device="cuda", nq=64, recipe="clustered", keep_outputs=False):
    """Eviction by accumulated attention weight beside the halving tree and uniform sampling, at equal numbers of kept tokens.  The first
    half of the queries of every head judges, the second half asks; errors are over the asking ones.  Eviction draws nothing: one run."""
    K, V, Q = make_inputs(device, n_seq=n_seq, n_mid=n_mid, nq=nq, recipe=recipe)
    n, d = K.shape[1], K.shape[2]
    judge, ask = Q[:, :, :nq // 2].contiguous(), Q[:, :, nq // 2:].contiguous()
    exact, _ = exact_attention_f64(K, V, ask)
    ones = torch.ones(n_seq, n, device=device)
    rows = []
    for T in rounds:
        acc = dict(tree=[], uniform=[], tree_ms=[], evict_ms=[])
        for s in range(seeds + 1):                          # run 0 warms up and is not counted
            p = binding.make_params(d, block, T, K.dtype, log_c=log_c_for(recipe, block), seed=1000 + s, center=True)
            ev = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
            ev[0].record()
            tree = binding.merge_reduce_protected(p, K, V, N_SINK, N_RECENT)
            ev[1].record()
            mass = binding.attend_mass(p, K, V, ones, judge)[2]
            heavy = binding.evict(p, K, V, ones, mass, tree["K"].shape[1], n_sink=N_SINK, n_recent=N_RECENT)
            ev[2].record()
            z, _ = binding.attend_kv(p, tree["K"], tree["V"], tree["w"], ask)
            ze, _ = binding.attend_kv(p, heavy["K"], heavy["V"], heavy["w"], ask)
            idx_u, w_u = uniform_sample_protected(n_seq, n, N_SINK, N_RECENT, T, 7000 + s, device)
            gi = idx_u[..., None].expand(-1, -1, d)
            zu, _ = binding.attend_kv(p, torch.gather(K, 1, gi), torch.gather(V, 1, gi), w_u, ask)
            torch.cuda.synchronize()
            if s == 0:
                continue
            acc["tree"].append(relative_error(z, exact)); acc["uniform"].append(relative_error(zu, exact))
            acc["tree_ms"].append(ev[0].elapsed_time(ev[1])); acc["evict_ms"].append(ev[1].elapsed_time(ev[2]))
        m = {k: float(torch.tensor(v).mean()) for k, v in acc.items()}
        m.update({k + "_std": _std(torch.tensor(acc[k])) for k in ("tree", "uniform")})
        m.update(rate="1/%d" % (1 << T), block=block, kept=int(tree["K"].shape[1]), evict=relative_error(ze, exact))
        if keep_outputs:
            m["last"] = dict(mass=mass, idx=heavy["idx"], w=heavy["w"], z=ze)
        rows.append(m)
    return dict(workload="%d KV sequences x (%d + %d + %d) tokens, d=%d, %d x %d judging and as many asking queries, bf16, synthetic (recipe %s)"
                         % (n_seq, N_SINK, n_mid, N_RECENT, d, Q.shape[1], judge.shape[2], recipe), seeds=seeds, rows=rows,
                **(dict(K=K, V=V, judge=judge, ask=ask, exact=exact) if keep_outputs else {}))


def evict_table(result):
    lines = ["| block | rate | kept | tree ms | mass + evict ms | BalanceKV rel. err | eviction rel. err | uniform rel. err |", "|---|---|---|---|---|---|---|---|"]
    for r in result["rows"]:
        lines.append("| %d | %s | %d | %.3f | %.3f | %.4f ± %.4f | %.4f | %.4f ± %.4f |"
                     % (r["block"], r["rate"], r["kept"], r["tree_ms"], r["evict_ms"], r["tree"], r["tree_std"], r["evict"], r["uniform"], r["uniform_std"]))
    return "\n".join(lines)


def alg1_table(result):
    lines = ["| block | rate | kept (numerator / denominator set) | build sets ms | two-set attend ms | Alg. 1 rel. err | one keys-only set | uniform |",
             "|---|---|---|---|---|---|---|---|"]
    for r in result["rows"]:
        lines.append("| %d | %s | %.0f / %.0f | %.3f | %.3f | %.4f ± %.4f | %.4f ± %.4f | %.4f ± %.4f |"
                     % (r["block"], r["rate"], r["kept_num"], r["kept_den"], r["sets_ms"], r["attend_ms"], r["alg1"], r["alg1_std"],
                        r["single"], r["single_std"], r["uniform"], r["uniform_std"]))
    return "\n".join(lines)


def as_table(result):
    lines = ["| block | rate | kept | compress ms | BalanceKV rel. err | uniform rel. err | BalanceKV normaliser err | uniform normaliser err |",
             "|---|---|---|---|---|---|---|---|"]
    for c in result["cells"]:
        lines.append("| %d | %s | %d | %.3f | %.4f ± %.4f | %.4f ± %.4f | %.5f ± %.5f | %.5f ± %.5f |"
                     % (c["block"], c["rate"], c["kept"], c["compress_ms"], c["balancekv_rel_err"], c["balancekv_std"],
                        c["uniform_rel_err"], c["uniform_std"], c["balancekv_normaliser_err"], c["balancekv_normaliser_std"],
                        c["uniform_normaliser_err"], c["uniform_normaliser_std"]))
    return "\n".join(lines)


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--seeds", type=int, default=10)
    ap.add_argument("--json", action="store_true", help="print one JSON line instead of the table")
    ap.add_argument("--value-factor", action="store_true", help="kernel weights times <v_i,v_j>/r_value^2 (Alg. 2 line 6)")
    ap.add_argument("--value-augment", action="store_true", help="kernel weights times (<v_i,v_j>/r_value^2 + 1) / 2: the value [v / r ; 1]")
    ap.add_argument("--alg1", action="store_true", help="Alg. 1 as listed (buckets, two kept sets) on heavy-tailed value norms")
    ap.add_argument("--evict", action="store_true", help="eviction by accumulated attention weight beside the tree and uniform sampling")
    ap.add_argument("--recipe", default="clustered", choices=["clustered", "iid"], help="input recipe of the grid")
    args = ap.parse_args(argv)
    if not torch.cuda.is_available():
        print("ablation: needs a GPU", file=sys.stderr)
        return 2
    binding.lib()
    if args.alg1:
        result = run_alg1(seeds=args.seeds)
        print(json.dumps(result) if args.json else result["workload"] + ", %d seeds\n" % result["seeds"] + alg1_table(result))
        return 0
    if args.evict:
        result = run_evict(seeds=args.seeds, recipe=args.recipe)
        print(json.dumps(result) if args.json else result["workload"] + ", %d seeds\n" % result["seeds"] + evict_table(result))
        return 0
    result = run(seeds=args.seeds, value_gram=args.value_factor, recipe=args.recipe, value_augment=args.value_augment)
    if args.json:
        print(json.dumps(result))
    else:
        print(result["workload"] + ", %d seeds" % result["seeds"])
        print(as_table(result))
    return 0


if __name__ == "__main__":
    sys.exit(main())
