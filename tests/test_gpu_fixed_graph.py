"""apar_decode_attention_fixed captured into a graph, as a pool's first fixed call, and replayed between eager calls (GPU only)."""
import pytest

import paper_2401_06761_amd as ap

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "bf16_fp8kv", "bf16_fp4kv"])
@pytest.mark.parametrize("n_q,n_kv,prompts,kids", [(8, 2, [300], 5), (8, 2, [9000], 4), (4, 4, [200] * 20, 3)])
def test_replays_equal_eager_calls(dtype, n_q, n_kv, prompts, kids):
    import torch

    gen = torch.Generator(device="cuda:0").manual_seed(3)
    with ap.Pool(n_q, n_kv, 128, dtype, 2000) as pool:
        h = pool.handle

        def rows(n, heads):
            return torch.randn((n, heads, 128), generator=gen, device="cuda:0").to(pool.torch_dtype)

        live = []
        for n in prompts:
            root = ap.apar_thread_create(h)
            ap.apar_append_kv(h, root, rows(n, n_kv), rows(n, n_kv))
            for kid in ap.apar_fork(h, root, kids):
                ap.apar_append_kv(h, kid, rows(3 + kid % 30, n_kv), rows(3 + kid % 30, n_kv))
                live.append(kid)
        q = rows(len(live), n_q)
        out, want = torch.zeros_like(q), torch.empty_like(q)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ap.apar_decode_attention_fixed(h, q, live, out)
        for _ in range(4):
            q.copy_(rows(len(live), n_q))
            out.zero_()
            graph.replay()
            ap.apar_decode_attention(h, q, live, want)
            torch.cuda.synchronize()
            assert torch.isfinite(want).all() and want.abs().max() > 0
            # (the same kernels; a plan whose cut does not fit the workspace is walked whole: equal to the outputs' roundings)
            if not torch.equal(out, want):
                top = float(want.abs().max())
                assert float((out.float() - want.float()).abs().max()) <= (1e-5 if dtype == "f32" else 2.0 ** -7) * top
