"""Calls of the cache operators that once gave wrong results, wrong errors or none."""
import numpy as np
import pytest

from paper_2601_11553_b200 import percache as pcb

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("n_seqs,ctx,hkv", [(1, 700, 1), (16, 2500, 8)])
@pytest.mark.parametrize("nodes", [1, 20])
def test_many_small_fp16_weights_are_not_lost(nodes, n_seqs, ctx, hkv):
    """Two slots (one in a block of each parity) have a score of 17.5 and values of 0, all others a score of 0 and values of 1000,
    so an output is 1000 n / (2 e^17.5 + n): each of the n weights is below 2^-25 of the largest, together they are the output.

    Tolerance.  Scores are exact.  An exponential and a row sum are off by 2^-19 relative, rounding to fp16 by 2^-11 of a weight, plus
    2^-32 of the largest where the weight is subnormal (multiples of 2^-24, the largest weight at 2^7 or more); the output is
    rounded once more (2^-11 relative; 2^-25 where it is subnormal)."""
    q_heads, d = 2 * hkv, 128
    t = ctx + nodes
    k = torch.zeros((n_seqs * t, hkv, d), dtype=torch.float16, device="cuda")
    v = torch.full((n_seqs * t, hkv, d), 1000.0, dtype=torch.float16, device="cuda")
    for b in range(n_seqs):
        for s in (3, 130):
            k[b * t + s, :, 0] = 17.5
            v[b * t + s] = 0.0
    q = torch.zeros((n_seqs * nodes, q_heads, d), dtype=torch.float16, device="cuda")
    q[:, :, 0] = 1.0
    out = torch.full_like(q, 7.0)
    lse = torch.zeros((n_seqs * nodes, q_heads), device="cuda")
    ws = torch.zeros(pcb.OPS_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    pcb.tree_attention(q, k, v, out, lse, ctx_len=torch.full((n_seqs,), ctx, dtype=torch.int32, device="cuda"),
                       row_start=torch.arange(0, n_seqs * nodes + 1, nodes, dtype=torch.int32, device="cuda"),
                       ctx_start=torch.arange(0, n_seqs * t, t, dtype=torch.int32, device="cuda"), max_nodes=nodes, max_len=t,
                       scale=1.0, workspace=ws)
    pcb.ops_status(ws)
    got = out.double().cpu().numpy().reshape(n_seqs, nodes, q_heads, d)
    for i in range(nodes):                                  # node i sees ctx + i + 1 slots
        n = ctx + i + 1 - 2
        total = 2 * np.exp(17.5) + n
        want = 1000.0 * n / total
        tol = (2.0 ** -10 + 2.0 ** -18) * want + 1000.0 * n * 2.0 ** -32 + 2.0 ** -25
        assert np.abs(got[:, i] - want).max() <= tol, (i, want, np.abs(got[:, i] - want).max(), tol)
        assert np.abs(lse.view(n_seqs, nodes, q_heads)[:, i].double().cpu().numpy() - np.log(total)).max() <= 2.0 ** -19 * 18


def small_handle(n_prompts, n_layers, reserve, **kw):
    """A handle after a prefill of n_prompts equal prompts of one token each."""
    from paper_2601_11553_b200 import workloads as wl
    shape = wl.ModelShape(n_layers=n_layers, d_model=256, n_q_heads=4, n_kv_heads=2, head_dim=128, d_ffn=512)
    weights = wl.make_weights(shape, 5, random_gains=True)
    h = pcb.PerCache(n_layers=n_layers, d_model=256, n_q_heads=4, n_kv_heads=2, head_dim=128, d_ffn=512, weights=weights, pool_pages=16,
                     max_prompt_tokens=1 + reserve, max_batch_prompts=n_prompts, max_batch_ctx_tokens=n_prompts * (1 + reserve),
                     max_batch_new_rows=n_prompts * 4, rope_theta=shape.rope_theta, rms_eps=shape.rms_eps, flags=pcb.FLAG_TRACK_WEIGHTS, **kw)
    h.set_decode_reserve(reserve)
    one = wl.make_hidden(5, (1,), 1, 256)
    h.prefill([pcb.PromptSpec([], [], [], one, 1) for _ in range(n_prompts)])
    return h, wl.make_hidden(5, (2,), 1, 256)


def test_running_weights_of_more_layers_and_prompts_than_a_grid_has_rows():
    n = 65535 // 28 + 1                                     # 28 layers: 65 548 lists of two heads
    h, token = small_handle(n, 28, 3)
    with h:
        tokens = np.ascontiguousarray(np.repeat(token, n, axis=0))
        h.decode_tree([[-1, -1]] * n, np.ascontiguousarray(np.repeat(token, 2 * n, axis=0)))
        h.accept([[1]] * n)              # moves the second node's weight to the first one's slot, and clears its own
        h.decode(tokens)                 # this token takes the slot that was cleared
        for layer in (0, 27):
            for b in (0, n - 1):
                w = h.read_weights(b, layer, 3, 2)
                # two rows, two heads a KV head.  A weight is off by its exponent's error: 2^-22 (|score| + |lse|), both far below 16
                assert np.abs(w.sum(1) - 4.0).max() <= 4 * 2.0 ** -17, (layer, b, w)
        h.evict_context(1)
        assert h.read_weights(n - 1, 27, 1, 2).shape == (2, 1)


def test_more_prompts_than_the_moves_can_take_are_refused_before_anything_runs():
    h, token = small_handle(65536, 1, 2)
    with h:
        tokens = np.ascontiguousarray(np.repeat(token, 65536, axis=0))
        for call in (lambda: h.decode_tree([[-1]] * 65536, tokens), lambda: h.decode(tokens)):
            with pytest.raises(pcb.PerCacheError) as e:
                call()
            assert e.value.code == pcb.E_CAPACITY
        h.set_flags(0)
        h.decode(tokens)                                    # plain steps go on


def leave_an_error_behind(h, token):
    """A decode step on a stream that is being captured is refused by the runtime (a host-side error; nothing runs)."""
    import ctypes as C
    cu = C.CDLL("libcuda.so.1")
    side = C.c_void_p(h.test_stream.cuda_stream)
    assert cu.cuStreamBeginCapture_v2(side, 2) == 0
    try:
        with pytest.raises(pcb.PerCacheError) as e:
            h.decode(token)
        assert e.value.code == pcb.E_CUDA
    finally:
        graph = C.c_void_p()
        cu.cuStreamEndCapture(side, C.byref(graph))
        if graph.value:
            cu.cuGraphDestroy(graph)


def handle_on_a_stream():
    side = torch.cuda.Stream()
    h, token = small_handle(1, 1, 12, stream=side.cuda_stream)
    h.test_stream = side
    h.decode(token)                                         # memory that the first step takes is there
    return h, token


def test_selection_and_moves_report_their_own_launch_only():
    h, token = handle_on_a_stream()
    with h:
        w = torch.rand((1, 2, 100), device="cuda")
        length = torch.tensor([100], dtype=torch.int32).cuda()
        keep = torch.empty((1, 2, 10), dtype=torch.int32, device="cuda")
        count = torch.empty(1, dtype=torch.int32, device="cuda")
        k = torch.randn((100, 2, 128), device="cuda").half()
        start = torch.zeros(1, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        leave_an_error_behind(h, token)
        pcb.select_slots(w, length, keep, count)
        leave_an_error_behind(h, token)
        pcb.compact_slots(k, k.clone(), keep, count, max_len=100, ctx_start=start)
        torch.cuda.synchronize()
        assert sorted(keep[0, 0].tolist()) == sorted(torch.topk(w[0, 0], 10).indices.tolist())


def test_steps_on_a_handle_report_their_own_errors_only():
    h, token = handle_on_a_stream()
    with h:
        leave_an_error_behind(h, token)
        h.decode(token)
        leave_an_error_behind(h, token)
        h.decode_tree([[-1, 0]], np.ascontiguousarray(np.repeat(token, 2, axis=0)))
        # (a step that fails drops the nodes, so the error before accept comes from another handle)
        other, t = handle_on_a_stream()
        with other:
            leave_an_error_behind(other, t)
            h.accept([[0, 1]])
            leave_an_error_behind(other, t)
            h.evict_context(2)
        h.decode(token)


def test_calls_without_a_stream_take_the_current_one():
    n, h = 200, 2
    gen = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)          # noqa: E731
    ints = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()                               # noqa: E731
    q, k, v = rnd(1, 4, 128), rnd(n, h, 128), rnd(n, h, 128)
    ws = torch.zeros(pcb.OPS_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    kw = dict(ctx_len=ints(n - 1), row_start=ints(0, 1), ctx_start=ints(0), max_nodes=1, max_len=n, workspace=ws)
    start = ints(0)

    def steps(q, k, v, wait):
        """Every operator on inputs that the current stream only has after `wait`."""
        out, lse = torch.zeros_like(q), torch.zeros((1, 4), device="cuda")
        w, w2 = torch.zeros((1, h, n), device="cuda"), torch.zeros((1, h, n), device="cuda")
        keep, count = torch.full((1, h, 50), -1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        qq, kk, vv, length = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), ints(0)
        torch.cuda.synchronize()
        wait()
        qq.copy_(q), kk.copy_(k), vv.copy_(v), length.fill_(n)
        pcb.tree_attention(qq, kk, vv, out, lse, **kw)
        wait()
        pcb.attention_weights(qq, kk, lse, w, w2, **kw)
        wait()
        pcb.select_slots(w2, length, keep, count, sink=1, recent=3)
        wait()
        pcb.compact_slots(kk, vv, keep, count, max_len=n, weights=w2, ctx_start=start)
        torch.cuda.synchronize()
        return out, lse, w2, keep, count, kk, vv

    want = steps(q, k, v, lambda: None)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = steps(q, k, v, lambda: torch.cuda._sleep(20_000_000))
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_the_status_of_a_workspace_is_read_behind_the_current_stream():
    ws = torch.zeros(pcb.OPS_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    pcb.ops_status(ws)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        ws[:4] = 1                                          # as a kernel does whose wait ran out
        with pytest.raises(pcb.PerCacheError) as e:
            pcb.ops_status(ws)
    assert e.value.code == pcb.E_DEVICE_TIMEOUT
    with pytest.raises(pcb.PerCacheError):
        pcb.ops_status(ws)
    ws[:4] = 0
    pcb.ops_status(ws)
