"""The operators around the routed experts under stream capture: a graph of all of them, replayed several times with eager work and
synchronizations in between, gives what the eager calls give."""
import pytest
import torch

from paper_2604_02715_amd import moe_block as M

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E,K,H", [(1, 512, 10, 2048), (300, 8, 2, 256), (3000, 160, 8, 520)])
def test_captured_calls_replay_as_the_eager_ones(T, E, K, H):
    g = torch.Generator(device="cuda").manual_seed(T)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    logits, residual, w = rand(T, E), rand(T, H), 1 + 0.1 * rand(H)
    rows_n = M.sorted_rows(T, K, E, 4)
    bf16 = lambda t: t.to(torch.bfloat16)

    def buffers():
        e = lambda *s: torch.full(s, float("nan"), device="cuda")
        return dict(ids=torch.zeros(T, K, **i32), gates=e(T, K), offsets=torch.zeros(E + 1, **i32), counts=torch.zeros(E, **i32),
                    pair_row=torch.zeros(T, K, **i32), row_pair=torch.zeros(rows_n, **i32), rows=bf16(e(rows_n, H)), out=e(T, H),
                    stream=e(T, H), normed=bf16(e(T, H)), d_rows=bf16(e(rows_n, H)), d_gates=e(T, K), d_logits=e(T, E), d_residual=e(T, H),
                    d_y=e(T, H), d_w=e(H), d_w_post=e(H),
                    sort_ws=torch.empty(M.sort_workspace_bytes(T, K, E), dtype=torch.uint8, device="cuda"),
                    grad_ws=torch.empty(M.block_norm_grad_workspace_bytes(T, H), dtype=torch.uint8, device="cuda"))

    def calls(b, x):
        M.route(logits, b["ids"], b["gates"])
        M.sort_tokens(b["ids"], E, b["offsets"], b["counts"], b["pair_row"], b["row_pair"], b["sort_ws"], align=4)
        M.dispatch(x, b["pair_row"], b["row_pair"], b["rows"])
        M.combine(b["rows"], b["pair_row"], b["gates"], b["out"])
        M.block_norm(residual, w, b["normed"], y=b["out"], w_post=w, residual_out=b["stream"])
        M.block_norm_grad(b["stream"], w, b["normed"], b["d_residual"], b["d_w"], b["grad_ws"], d_residual_out=residual, y=b["out"], w_post=w,
                          d_y=b["d_y"], d_w_post=b["d_w_post"])
        M.combine_grad(b["d_y"], b["rows"], b["pair_row"], b["row_pair"], b["gates"], b["d_rows"], b["d_gates"])
        M.route_grad(logits, b["ids"], b["d_gates"], b["d_logits"])

    x = bf16(rand(T, H))
    eager, captured = buffers(), buffers()
    calls(eager, x)
    torch.cuda.synchronize()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        calls(captured, x)
    for turn in range(4):
        x.copy_(bf16(rand(T, H)))                            # eager work and new inputs between the replays
        logits.copy_(rand(T, E))
        calls(eager, x)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in eager:
            if not name.endswith("_ws"):
                assert torch.equal(eager[name], captured[name]), (turn, name)
