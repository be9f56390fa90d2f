"""The operators of a model's step together, as a server runs them: rotary positions, a 4-bit pool, prefill and decode attention, logits, draws,
Alg. 1.  Every step's output is held to a plain computation in 64 bits on what the step was given."""
import numpy as np
import pytest

import paper_2401_06761_amd as ap
from apar_workloads import EOS, FORK, SamplerConfig, make_requests, uniforms
from oracle import DenseThreads, attend, fp4, sampling
from oracle.controller import SequenceGroup
from paper_2401_06761_amd.serving import ServingRun

from harness import to_host
from test_gpu_fp4kv import assert_within
from test_gpu_rotary import check as check_rotated

pytestmark = pytest.mark.gpu
CONTROL = {-1: 0, -2: 1, -3: 2}


def check_draw(x, cuts, u, token, ids):
    """x: a row of logits on the host.  A draw that is a tie of the sums is not told apart (none has been met)."""
    want, _, margin = sampling.draw(x, np.float32(cuts[0]), int(cuts[1]), np.float32(cuts[2]), np.float32(cuts[3]), np.float32(u))
    got = ids[CONTROL[int(token)]] if token in CONTROL else int(token)
    assert got == want or margin <= 2.0 ** -(62 - 2 * int(np.ceil(np.log2(len(x))))) + 1e-12, (got, want, margin)


@pytest.mark.parametrize("n_q,n_kv,layout", [(8, 2, "half"), (4, 4, "pairs")])
def test_groups_of_a_small_model(n_q, n_kv, layout):
    import torch

    rng = np.random.default_rng(31)
    gen = torch.Generator(device="cuda:0").manual_seed(31)
    vocab, dim, d = 203, 64, 128
    ids = (vocab - 3, vocab - 2, vocab - 1)

    def weights(*shape, scale=1.0):
        return scale * torch.randn(shape, generator=gen, device="cuda:0")

    table, wq, wk, wv = weights(vocab, dim), *(weights(dim, n * d, scale=dim ** -0.5) for n in (n_q, n_kv, n_kv))
    head = weights(n_q * d, vocab, scale=0.1)

    def project(tokens, w, heads):
        index = [ids[CONTROL[x]] if x in CONTROL else x for x in tokens]
        return (table[torch.tensor(index, device="cuda:0")] @ w).bfloat16().view(-1, heads, d)

    def new_rows(rot, tokens, positions):
        """K at its positions, and V, of tokens to be appended; K checked."""
        k, v = project(tokens, wk, n_kv), project(tokens, wv, n_kv)
        turned = torch.empty_like(k)
        ap.apar_rotate_rows(rot.handle, torch.tensor(positions, dtype=torch.int32, device="cuda:0"), None, k, None, turned)
        check_rotated(turned, k, positions, rot)
        return turned, v

    with ap.Pool(n_q, n_kv, d, "bf16_fp4kv", 400) as pool, ap.Rotary(d, 96, layout) as rot:
        ap.apar_set_write_checks(pool.handle, True)
        pool.kv.fill_(0xFF)
        dense = DenseThreads(n_q, n_kv, d)
        groups = []
        for n in (1, 16, 75):
            prompt = [int(x) for x in rng.integers(0, vocab - 3, n)]
            k, v = new_rows(rot, prompt, list(range(n)))
            grp, o = ap.apar_group_create(pool.handle, prompt, k, v), SequenceGroup(prompt)
            tid = {0: ap.apar_group_unfinished(grp)[0]}
            assert dense.create() == tid[0]
            dense.append(tid[0], fp4.held(to_host(k)), fp4.held(to_host(v)))
            groups.append((grp, o, tid))
        # the prompts' own rows attend to each other
        roots = [tid[0] for _, _, tid in groups]
        m = [len(o.G[0].tokens) for _, o, _ in groups]
        q = torch.cat([project(o.G[0].tokens, wq, n_q) for _, o, _ in groups])
        turned, out = torch.empty_like(q), torch.empty_like(q)
        ap.apar_rotate_threads(pool.handle, rot.handle, roots, q, None, turned, m=m, where=ap.APAR_ROWS_LAST)
        check_rotated(turned, q, [j for n in m for j in range(n)], rot)
        ap.apar_prefill_attention(pool.handle, turned, roots, m, out)
        at = 0
        for root, n in zip(roots, m):
            K, V = dense._get(root)
            want = np.stack([attend(to_host(turned)[at + j], K[:j + 1], V[:j + 1], d ** -0.5) for j in range(n)])
            assert_within(to_host(out)[at:at + n], want, np.abs(V).max(), f"prompt of {n}")
            at += n

        forks = ends = 0
        for step in range(60):
            todo = [(g, s) for g in groups for s in g[1].unfinished()]
            if not todo:
                break
            live = [g[2][s.sid] for g, s in todo]
            assert live == [t for grp, _, _ in groups for t in ap.apar_group_unfinished(grp)]
            q = project([s.last_token for _, s in todo], wq, n_q)
            turned, out = torch.empty_like(q), torch.empty_like(q)
            ap.apar_rotate_threads(pool.handle, rot.handle, live, q, None, turned, where=ap.APAR_ROWS_LAST, m=[1] * len(live))
            check_rotated(turned, q, [len(s.tokens) - 1 for _, s in todo], rot)
            ap.apar_decode_attention(pool.handle, turned, live, out)
            top_v = max(np.abs(dense._get(th)[1]).max() for th in live)
            assert_within(to_host(out), dense.decode(to_host(turned), live), top_v, f"step {step}")

            logits = out.float().view(len(live), -1) @ head
            logits[:, ids[0]] += torch.tensor([-30.0 if s.last_token == FORK or len(g[1].G) > 5 else 3.0 for g, s in todo], device="cuda:0")
            logits[:, ids[1]] = -float("inf")
            logits[:, ids[2]] += 2.0 if step > 20 else -30.0
            u = rng.random(len(live)).astype(np.float32)
            cuts = [(0.7 + 0.1 * (i % 7), 20 * (i % 3), 0.5 + 0.1 * (i % 6), 0.01 * (i % 2)) for i in range(len(live))]
            rows = ap.apar_sample_rows(*(torch.tensor([c[j] for c in cuts], device="cuda:0") for j in range(4)))
            tokens = torch.empty(len(live), dtype=torch.int32, device="cuda:0")
            ap.apar_sample_tokens(logits, torch.from_numpy(u).cuda(), tokens, rows, token_ids=ids)
            sampled, host = tokens.tolist(), logits.cpu().numpy()
            for i in range(len(live)):
                check_draw(host[i], cuts[i], u[i], sampled[i], ids)
            for grp, o, tid in groups:
                mine = [i for i, (g, _) in enumerate(todo) if g[1] is o]
                if not mine:
                    continue
                xs = [sampled[i] for i in mine]
                forkers, before = [s for s in o.unfinished() if s.last_token == FORK], len(o.G)
                appended = o.step(xs)  # (a row each; a sequence that forks has its child's row before its own)
                places = [len(s.tokens) - 1 for s in appended]
                k, v = new_rows(rot, [s.tokens[-1] for s in appended], places)
                assert ap.apar_group_step(grp, xs, k, v).n_rows_appended == len(appended)
                for s, c in zip(forkers, o.G[before:]):
                    (tid[c.sid],) = dense.fork(tid[s.sid], 1)
                for i, s in enumerate(appended):
                    dense.append(tid[s.sid], fp4.held(to_host(k)[i:i + 1]), fp4.held(to_host(v)[i:i + 1]))
                for s in o.G:
                    if s.finished and tid[s.sid] in dense._k:
                        dense.free(tid[s.sid])
                        ends += 1
                forks += len(forkers)
        assert forks > 0 and ends > 0
        for grp, o, _ in groups:
            assert ap.apar_group_restore(grp) == o.restore()
            ap.apar_group_destroy(grp)
        st = ap.apar_pool_stats(pool.handle)
        assert st.live_threads == 0 and st.free_blocks == st.total_blocks


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_serving_loop_draws_from_logits(dtype):
    """Requests that fork, end and are preempted; every token is the one that the definition draws from the step's logits."""
    import torch

    n_q, n_kv, d, vocab = 4, 2, 128, 611
    cfg = SamplerConfig(vocab=vocab, max_threads=6, min_new=10, max_len=140)
    ids, cuts = (600, 601, 602), (0.9, 200, 0.95, 0.001)
    gen = torch.Generator(device="cuda:0").manual_seed(7)
    q, k, v = (torch.randn((n, h, d), generator=gen, device="cuda:0").bfloat16() for n, h in ((64, n_q), (512, n_kv), (512, n_kv)))
    head = 0.2 * torch.randn((n_q * d, vocab), generator=gen, device="cuda:0")
    head[:, [600, 602]] = 0.0
    bias = torch.zeros(vocab, device="cuda:0")
    bias[600], bias[602] = 3.5, 3.0
    steps = []

    def logits(batch, out):
        x = (out.float().view(len(batch), -1) @ head + bias).to(torch.float32 if dtype == "f32" else torch.bfloat16)
        steps.append((batch, x))
        return x

    reqs = make_requests(8, seed=5, prompt_lo=8, prompt_hi=60)
    seeds = {r.rid: r.seed for r in reqs}
    with ap.Pool(n_q, n_kv, d, "bf16_fp4kv", 48, max_threads=1 << 20) as pool:
        run = ServingRun(pool, reqs, cfg, 6, 1, banks=(q, k, v), logits=logits, token_ids=ids, cuts=cuts)
        run.keep_trace = True
        st = run.run()
        run.close()
    assert st["finished"] == 8 and len(steps) == len(run.trace) == st["steps"]
    assert st["preemptions"] > 0 and sum(t["n_forked"] for t in run.trace) > 0
    for (batch, x), t in zip(steps, run.trace):
        host = x.float().cpu().numpy()
        u = uniforms([seeds[int(r)] for r in batch["request_id"]], batch["seq_index"], batch["length"])
        assert np.isneginf(host[:, 601]).all()
        for i in range(len(batch)):
            if batch["length"][i] + 1 >= cfg.max_len:
                assert t["sampled"][i] == EOS
            else:
                check_draw(host[i], cuts, u[i], t["sampled"][i], ids)


def test_the_serving_loop_refuses_logits_without_what_they_need():
    reqs = make_requests(1)
    with ap.Pool(4, 2, 128, "bf16", 64, dry_run=True) as pool:
        for bad in ({}, {"token_ids": (1, 2, 3)}):
            with pytest.raises(ValueError):
                ServingRun(pool, reqs, SamplerConfig(), 2, 0, logits=lambda b, o: o, **bad)
