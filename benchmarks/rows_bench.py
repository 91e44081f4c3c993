"""Times the entry points that widen the hot path, at the 8B shape (V = 128256, k = 10, 61 tree rows):
acceptance-length distribution, prediction-model step (alone and fused into the expansion), the
expansion of 4, 16 and 64 sequences in one launch, verification with draft distributions, the paged 4-bit cache, and prompts and tokens over it.  One JSON line per entry point with the per-kernel device
durations the library records (radar_profile_begin / radar_profile_end) and the algorithmic bytes.

    python -m benchmarks.rows_bench [--reps 100]
"""
import argparse
import json
import sys


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--reps", type=int, default=100)
    args = ap.parse_args()
    import numpy as np
    import torch
    from paper_2512_14069_amd import binding as b, synth

    if not torch.cuda.is_available():
        print("rows_bench: no GPU visible", file=sys.stderr)
        sys.exit(1)
    dev = "cuda"
    c3 = synth.config(3)
    V, k, N = c3.vocab, c3.k, c3.N
    T = N + 1
    rng = np.random.default_rng(synth.seed_for(3, 91))
    to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)

    def timed(name, calls, bytes_per_call, note):
        for _ in range(10):
            for c in calls:
                c()
        torch.cuda.synchronize()
        b.radar_profile_begin(args.reps * len(calls) * 4)
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        for _ in range(args.reps):
            for c in calls:
                c()
        kern = b.radar_profile_end()
        e0.record()
        for _ in range(args.reps):
            for c in calls:
                c()
        e1.record()
        torch.cuda.synchronize()
        us = e0.elapsed_time(e1) * 1e3 / args.reps
        print(json.dumps({"entry": name, "us_back_to_back": round(us, 2), "algorithmic_bytes": int(bytes_per_call),
                          "GBps_back_to_back": round(bytes_per_call / us / 1e3, 1),
                          "kernels_us": {n: round(v["mean_us"], 2) for n, v in kern.items()}, "note": note}), flush=True)

    # trees of the verify shape with sampled tokens
    par = [synth.make_tree(rng, T, 8, k, V)[0]]
    x = synth.sampled_draft_inputs(rng, par, V, T, std=2.0, noise=1.0, shared_rows=True)
    d = {n: to(v) for n, v in x.items()}

    desc = b.accept_desc(1, T, V, T - 1, b.RADAR_ACCEPT_SAMPLE, 1.0)
    ws = b.new_workspace(b.radar_verify_accept_workspace_bytes(desc))
    call = b.radar_accept_length_distribution(d["target_logits"], d["draft_tokens"], d["parents"], d["n_nodes"],
                                              workspace=ws, prepared=True)
    timed("radar_accept_length_distribution", [call], T * V * 4, "bytes: 61 target rows, of which those of leaves are left unread")

    pw = synth.policy_params(rng, k)
    pp = b.policy_params({n: to(v) for n, v in pw.items()})
    pbytes = sum(v.nbytes for v in pw.values())
    conf = to(synth.policy_conf(rng, 1, k)[0])
    pout = b.PolicyOut(1, synth.POLICY_H, dev)
    call = b.radar_policy_step(conf, pp, pout.h, pout.c, out=pout, prepared=True)
    timed("radar_policy_step", [call], pbytes, "parameters read once (they stay in L2 between calls)")

    for F in (1, k):
        logits = to(synth.expand_logits(rng, F, V, c3.logit_std))
        ps, pi = torch.zeros(F, device=dev), torch.full((F,), -1, dtype=torch.int32, device=dev)
        pool = b.DraftPool(4096)
        ews = b.new_workspace(b.radar_draft_expand_workspace_bytes(b.expand_desc(F, V, k, 0, 4096)))
        eo = b.ExpandOut(F, k, dev)
        plain = b.radar_draft_expand(logits, ps, pi, k, pool, out=eo, workspace=ews, prepared=True)
        pool.count = 0
        fused = b.radar_draft_expand_policy(logits, ps, pi, k, pool, pp, pout.h, pout.c, out=eo, policy_out=pout,
                                            workspace=ews, prepared=True)
        pool.count = 0
        sep = b.radar_policy_step(eo.frontier_conf, pp, pout.h, pout.c, out=pout, prepared=True)
        timed("radar_draft_expand F=%d" % F, [plain], F * V * 4, "for comparison")
        timed("radar_draft_expand_policy F=%d" % F, [fused], F * V * 4 + pbytes, "expansion and decision in one launch")
        timed("radar_draft_expand + radar_policy_step F=%d" % F, [plain, sep], F * V * 4 + pbytes, "two launches")

    # one draft call for B sequences in one launch; inputs rotated through more memory than the caches hold
    gen = torch.Generator(device=dev)
    gen.manual_seed(synth.seed_for(3, 92))
    for B in (4, 16, 64):
        nsets = max(2, int(600e6 // (B * k * V * 4)) + 1)
        sets = [torch.log_softmax(torch.randn((B, k, V), generator=gen, device=dev) * c3.logit_std, dim=-1).contiguous()
                for _ in range(nsets)]
        ps = torch.zeros((B, k), device=dev)
        pi = torch.full((B, k), -1, dtype=torch.int32, device=dev)
        pool = b.DraftPool(k * k, B=B)
        bws = b.new_workspace(b.radar_draft_expand_batch_workspace_bytes(b.expand_desc(k, V, k, 0, k * k), B))
        eo = b.ExpandOut(k, k, dev, B=B)
        calls = []
        for lg in sets:
            pool.count = 0
            calls.append(b.radar_draft_expand_batch(lg, ps, pi, k, pool, out=eo, workspace=bws, prepared=True))
        # timed() runs the whole list per repetition: report per call
        args.reps, keep = max(1, args.reps // nsets), args.reps
        timed("radar_draft_expand_batch B=%d F=%d (%d calls)" % (B, k, nsets), calls, nsets * B * k * V * 4,
              "%d sequences per launch; time and bytes are for %d calls on different inputs" % (B, nsets))
        if B == 16:                                        # the same calls with the decision of every sequence in them
            poutB = b.PolicyOut(B, synth.POLICY_H, dev)
            poutB.h.zero_(); poutB.c.zero_()
            calls = []
            for lg in sets:
                pool.count = 0
                calls.append(b.radar_draft_expand_batch(lg, ps, pi, k, pool, params=pp, h=poutB.h, c=poutB.c, out=eo,
                                                        policy_out=poutB, workspace=bws, prepared=True))
            args.reps = max(1, keep // nsets)
            timed("radar_draft_expand_batch B=%d F=%d with the prediction model (%d calls)" % (B, k, nsets), calls,
                  nsets * (B * k * V * 4 + pbytes), "as above, with every sequence's continue / stop decision in the call")
        args.reps = keep
        del sets, calls
        torch.cuda.empty_cache()

    qd = b.accept_q_desc(1, T, T, V, T - 1)
    qws = b.new_workspace(b.radar_verify_accept_q_workspace_bytes(qd))
    for limit, label in ((0, "walk shared by 32 workgroups"), (-1, "walk by one workgroup")):
        call = b.radar_verify_accept_q(d["target_logits"], d["draft_logits"], d["draft_tokens"], d["parents"], d["n_nodes"],
                                       d["uniforms"], d["q_rows"], workspace=qws, prepared=True, walk_spin_limit=limit)
        used = len(set(x["q_rows"][0, 1:T].tolist()))
        timed("radar_verify_accept_q", [call], (T + used) * V * 4, label + "; bytes: %d target rows and %d draft rows, of which the shared walk reads those it visits" % (T, used))

    # the paged 4-bit cache of one layer: 32 heads on 8, D = 128; 2048 to 8192 rows of prefix
    Hq, H, D, R = 32, 8, 128, 16
    for B, Tq, lo, hi in ((1, 1, 2048, 2048), (64, 1, 2048, 8192), (1, 60, 2048, 2048), (16, 60, 2048, 8192)):
        L = rng.integers(lo, hi + 1, B)
        per = -(-(int(L.max()) + Tq) // R)
        n_blocks = sum(-(-(int(x) + Tq) // R) for x in L)
        cache, tables = b.KvqCache(n_blocks, R, H, D), b.KvqTables(B, per, n_blocks, R)
        cache.data.random_(0, 256, generator=gen)
        cache.data[..., R * D:].fill_(126)
        ctx = to(L.astype(np.int32))
        b.radar_kvq_blocks(torch.zeros_like(ctx), tables, int(L.max()), n_new=ctx)
        kv = torch.randn((2, B, Tq, H, D), generator=gen, device=dev).to(torch.bfloat16)
        q = torch.randn((B, Tq, Hq, D), generator=gen, device=dev).to(torch.bfloat16)
        parents = to(np.tile(synth.make_tree(rng, Tq, 8, k, V)[0], (B, 1)).astype(np.int32)) if Tq > 1 else None
        room = b.radar_kvq_blocks(ctx, tables, Tq, prepared=True)
        room()
        write = b.radar_kvq_append(cache, kv[0], kv[1], room.out[0], prepared=True)
        what = "B=%d T=%d, %d rows of prefix" % (B, Tq, int(L.sum()))
        row = H * (D + D // 16)
        attend = b.radar_tree_attention_kvq(q, cache, tables.block_tables, ctx, parents, S_max=int(L.max()) + Tq, prepared=True)
        timed("radar_tree_attention_kvq " + what, [attend], (int(L.sum()) + B * Tq) * row + q.numel() * 4, "bytes: the sequences' rows once, queries and outputs")
        if Tq > 1:
            length, path = torch.full((B,), 6, dtype=torch.int32, device=dev), to(np.tile([0, 3, 9, 17, 30, 41, 55], (B, 1)).astype(np.int32))
            move = b.radar_kvq_commit(cache, tables.block_tables, ctx, length, path, prepared=True)
            timed("radar_kvq_blocks + append + commit " + what, [room, write, move], B * Tq * (4 * H * D + row) + B * 6 * 2 * row,
                  "a verification pass's other calls; bytes: the trees' rows in and the paths' rows")
        del cache
        torch.cuda.empty_cache()

    # serving steps over it: rows turned by their positions and written, and attention of the new rows (prompts, pieces of them, single tokens)
    rope = b.Rope((10000.0 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))).float().to(dev))
    for what, ctxs, news in (("a tree of 60 rows behind 2048", [2048], [60]), ("a prompt of 2048 rows", [0], [2048]), ("a prompt of 16384 rows", [0], [16384]),
                             ("512 rows behind 16384", [16384], [512]), ("64 tokens behind 2048 to 8192", rng.integers(2048, 8193, 64), [1] * 64),
                             ("48 tokens and two pieces of 400 rows behind 512 to 8192", rng.integers(512, 8193, 50), [1] * 48 + [400] * 2)):
        L, n = np.asarray(ctxs, np.int64), np.asarray(news, np.int64)
        B, rows, most = len(L), int(n.sum()), int(n.max())
        per, n_blocks = -(-int((L + n).max()) // R), int(sum(-(-int(x) // R) for x in L + n))
        cache, tables = b.KvqCache(n_blocks, R, H, D), b.KvqTables(B, per, n_blocks, R)
        cache.data.random_(0, 256, generator=gen)
        cache.data[..., R * D:].fill_(126)
        ctx, new, starts = to(L.astype(np.int32)), to(n.astype(np.int32)), to(np.concatenate([[0], np.cumsum(n)]).astype(np.int32))
        x = torch.randn((rows, Hq + 2 * H, D), generator=gen, device=dev).to(torch.bfloat16)
        q, kk, vv = x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]
        slots, _ = b.radar_kvq_blocks(ctx, tables, most, n_new=new)
        row, span = H * (D + D // 16), dict(ctx_lens=ctx, row_starts=starts)
        turn = b.radar_rope(q, kk, rope, T_max=most, prepared=True, **span)
        timed("radar_rope " + what, [turn], rows * (Hq + H) * D * 4, "q and k, in and out")
        write = b.radar_kvq_append_rope(cache, q, kk, vv, slots, rope, prepared=True, **span)
        timed("radar_kvq_append_rope " + what, [write], rows * (Hq * D * 4 + 4 * H * D + row), "q in and out, k and v in, the cache's rows out")
        attend = b.radar_chunk_attention_kvq(write.out, cache, tables.block_tables, T_max=most, S_max=int((L + n).max()), prepared=True, **span)
        flop = 4 * Hq * D * float((n * L + n * (n + 1) / 2).sum())
        timed("radar_chunk_attention_kvq " + what, [attend], int((L + n).sum()) * row + rows * Hq * D * 4,
              "bytes: the sequences' rows once, queries and outputs; %.3g Gflop" % (flop / 1e9))
        del cache, x
        torch.cuda.empty_cache()


if __name__ == "__main__":
    main()
