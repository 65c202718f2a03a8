"""Routing, exchange, products by expert and adapters as they run together: a layer's values and
gradients, serving with codes, captured steps, streams and threads.

Bound of the FP8 layers' relative error: 0.056 for one product, as in test_gpu_experts; the joins, the
weights and 16-bit roundings add less than 0.005, and the gradient of the logits, a product of the
layer's outputs and dout, has the outputs' error.
"""
from __future__ import annotations

import threading

import pytest
import torch

import tokens_reference as R
from paper_2412_08832_amd import hadacore as H

pytestmark = pytest.mark.gpu
REL = 0.061


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    H.library()
    yield
    torch.cuda.synchronize()


def _rel(got, want):
    return float((got.detach().double().cpu() - want).norm() / want.norm())


def _make(tokens, experts, n, k, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    x, w = torch.randn((tokens, k), generator=gen), torch.randn((experts, n, k), generator=gen) / k ** 0.5
    return x.to(dtype), torch.randn((tokens, experts), generator=gen), w.to(dtype)


def _plain(x, logits, w, k, renormalize, valid):
    chosen, weights, _, loss, _ = R.route(logits, k, renormalize, valid)
    y = torch.einsum("tk,enk->ten", x, w)
    picked = y.gather(1, chosen.clamp(min=0).long()[..., None].expand(-1, -1, w.shape[1]))
    return (picked * weights[..., None]).sum(1), loss, chosen


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tokens,experts,n,k,choices,renormalize,padded", [
    (300, 4, 96, 256, 2, True, False), (130, 9, 64, 512, 3, False, True), (1, 4, 32, 128, 1, True, False),
    (77, 16, 40, 384, 8, True, True)])
def test_mixture(tokens, experts, n, k, choices, renormalize, padded, dtype):
    from paper_2412_08832_amd import experts as E
    x, logits, w = _make(tokens, experts, n, k, dtype)
    valid = torch.rand(tokens, generator=torch.Generator().manual_seed(1)) > 0.3 if padded else None
    dy = torch.randn((tokens, n), generator=torch.Generator().manual_seed(2))
    wide = [t.double().requires_grad_() for t in (x, logits, w)]
    want, want_loss, chosen = _plain(*wide, choices, renormalize, valid)
    want_grads = torch.autograd.grad((want * dy.double()).sum() + 0.1 * want_loss, wide)
    leaves = [t.cuda().requires_grad_() for t in (x, logits, w)]
    on_gpu = None if valid is None else valid.cuda()
    out, routes = E.mixture(*leaves, choices, renormalize, on_gpu)
    assert torch.equal(routes.experts.cpu(), chosen)
    ((out.float() * dy.cuda()).sum() + 0.1 * routes.loss).backward()
    assert _rel(out, want.detach()) <= REL
    # as in test_gpu_route, for logits up to 8 apart
    assert abs(float(routes.loss.detach()) - float(want_loss.detach())) <= 496 * R.U * float(want_loss.detach())
    for name, leaf, ref in zip(("x", "logits", "w"), leaves, want_grads):
        if float(ref.norm()) > 0:
            assert leaf.grad.dtype == leaf.dtype and _rel(leaf.grad, ref) <= REL, name
    q = E.quantize_weights(leaves[2].detach(), backward=False)
    served = E.serve_mixture(leaves[0].detach(), leaves[1].detach(), q, choices, renormalize, on_gpu)
    assert torch.equal(served, out)
    if padded:
        assert (out[~on_gpu] == 0).all() and (leaves[0].grad[~on_gpu] == 0).all()


@pytest.mark.parametrize("wide", [False, True])
def test_adapters_beside_a_projection(wide):
    """The adapters' part beside an FP8 projection, in its type or 32 bits, and its gradients."""
    from paper_2412_08832_amd import adapters as A
    from paper_2412_08832_amd import experts as E
    gen = torch.Generator().manual_seed(0)
    x = torch.randn((200, 512), generator=gen).bfloat16()
    w = (torch.randn((96, 512), generator=gen) / 23).bfloat16()
    down, up = (torch.randn((3, 8, 512), generator=gen) / 23).bfloat16(), torch.randn((3, 8, 96), generator=gen).bfloat16()
    ids, dout = torch.randint(-1, 3, (200,), generator=gen).int(), torch.randn((200, 96), generator=gen).bfloat16()
    scales = torch.tensor([0.5, 1.0, 2.0])
    ends, _, slots = R.group(ids, 3)
    groups = H.group_tokens(ids.cuda(), 3)
    assert torch.equal(groups.ends.cpu(), ends) and torch.equal(groups.slots.cpu(), slots)
    leaves = [t.cuda().requires_grad_() for t in (x, down, up)]
    y = E.linear(leaves[0].detach(), E.quantize_weights(w.cuda(), backward=False))
    y = (y.float() if wide else y).requires_grad_()
    out = A.adapt(y, *leaves, groups, scales.cuda())
    assert out.dtype == y.dtype
    out.backward(dout.cuda().to(out.dtype))
    want, off, *_ = R.adapt(x, down, up, ends, slots, y.detach().cpu(), scales, *R.parts(torch.bfloat16, out.dtype))
    R.check("out", out, want, R.rounded(want, off, out.dtype))
    want, off, *_ = R.adapt(dout, up, down, ends, slots, None, scales, *R.parts(torch.bfloat16, torch.bfloat16))
    R.check("dx", leaves[0].grad, want, R.rounded(want, off, torch.bfloat16))
    assert torch.equal(y.grad, dout.cuda().to(y.dtype))
    for leaf, weight, rows, other in ((leaves[1], up, dout, x), (leaves[2], down, x, dout)):
        _, _, h, h_off = R.adapt(rows, weight, weight, ends, slots, None, None, 0, 0)
        ref, off = R.weight_gradient(h, other, ends, slots, scales, torch.bfloat16, torch.bfloat16)
        more, _ = R.weight_gradient(h_off, other.double().abs(), ends, slots, scales, torch.bfloat16, torch.bfloat16)
        R.check("weight", leaf.grad, ref, R.rounded(ref, off + more, torch.bfloat16))


def _serve(x, logits, q, down, up, ids, scales):
    """Router, experts and adapters, as one step of a server."""
    routes = H.route_tokens(logits, 2)
    groups = H.group_tokens(routes.experts, 8)
    a, sa = H.transform_fp8_blocks(x)
    y = H.grouped_matmul_fp8(H.dispatch_rows(a, groups.rows, groups.ends), H.dispatch_rows(sa, groups.rows, groups.ends),
                             q.codes, q.scales, groups.ends, dtype=x.dtype)
    out = H.combine_rows(y, groups.rows, routes.weights)
    plan = H.group_tokens(ids, down.shape[0])
    H.adapt_rows(x, down, up, plan.ends, plan.slots, y=out, scales=scales, out=out)
    return out, routes.counts, routes.loss


def _server(tokens):
    from paper_2412_08832_amd import experts as E
    x, logits, w = (t.cuda() for t in _make(tokens, 8, 256, 512, torch.bfloat16, seed=tokens))
    q = E.quantize_weights(w, backward=False)
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    down = (torch.randn((5, 16, 512), generator=gen, device="cuda") / 23).bfloat16()
    up = torch.randn((5, 16, 256), generator=gen, device="cuda").bfloat16()
    scales = torch.rand(5, generator=gen, device="cuda")
    ids = torch.randint(-1, 5, (tokens,), generator=gen, device="cuda").int()
    return x, logits, q, down, up, ids, scales


@pytest.mark.parametrize("tokens", [3, 64, 5000])
def test_captured_server_replays(tokens):
    """One step in a graph, replayed on new inputs between eager work; every replay is the eager result."""
    data = _server(tokens)
    x, logits, ids = data[0], data[1], data[5]
    _serve(*data)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            held = _serve(*data)
    torch.cuda.current_stream().wait_stream(side)
    gen = torch.Generator(device="cuda").manual_seed(9)
    for replay in range(4):
        x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        logits.copy_(torch.randn(logits.shape, generator=gen, device="cuda"))
        ids.copy_(torch.randint(-1, 5, ids.shape, generator=gen, device="cuda"))
        want = [t.clone() for t in _serve(*data)]
        for t in held:
            t.fill_(-7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), f"replay {replay}"


def _train(x, logits, dout, down, up, ids):
    """The calls of a training step by hand: everything that its backward pass launches."""
    routes = H.route_tokens(logits, 2, renormalize=False)
    groups = H.group_tokens(routes.experts, logits.shape[1])
    rows = H.dispatch_rows(x, groups.rows, groups.ends)
    out = H.combine_rows(rows, groups.rows, routes.weights)
    dy, dweights = H.combine_rows_gradient(dout, rows, groups.rows, groups.ends, routes.weights)
    dx = H.combine_rows(dy, groups.rows)
    dlogits = H.route_tokens_gradient(logits, routes, dweights, routes.loss)
    plan = H.group_tokens(ids, down.shape[0])
    adapted, h = H.adapt_rows(x, down, up, plan.ends, plan.slots, hidden=True)
    back, dh = H.adapt_rows(adapted, up, down, plan.ends, plan.slots, hidden=True)
    grads = (H.adapter_gradient(dh, x, plan.ends, plan.slots, dtype=torch.float32),
             H.adapter_gradient(h, adapted, plan.ends, plan.slots))
    return out, dy, dweights, dx, dlogits, adapted, back, *grads


def _trainer(tokens):
    gen = torch.Generator(device="cuda").manual_seed(tokens)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    return (normal(tokens, 384).half(), normal(tokens, 20), normal(tokens, 384).half(), (normal(4, 24, 384) / 20).half(),
            (normal(4, 24, 384) / 20).half(), torch.randint(-1, 4, (tokens,), generator=gen, device="cuda").int())


@pytest.mark.parametrize("tokens", [40, 4000])
def test_captured_training_calls_replay(tokens):
    data = _trainer(tokens)
    _train(*data)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            held = _train(*data)
    torch.cuda.current_stream().wait_stream(side)
    for replay in range(3):
        for t, new in zip(data, _trainer(tokens + 1 + replay)):
            t.copy_(new[: t.shape[0]])
        want = [t.clone() for t in _train(*data)]
        for t in held:
            t.fill_(-7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), f"replay {replay}"


def test_captured_backward():
    """A step of autograd in a graph: leaves of its own, the warm-up on the capture's stream and its
    graph gone before the capture."""
    from paper_2412_08832_amd import adapters as A
    from paper_2412_08832_amd import experts as E
    x, logits, dout, down, up, ids = _trainer(64)
    groups = H.group_tokens(ids, 4)

    def step(leaves):
        routes = E.route(leaves[1], 2)
        plan = H.group_tokens(routes.experts, 20)
        out = E.combine(E.dispatch(leaves[0], plan), plan, routes.weights)
        out = A.adapt(out, leaves[0], leaves[2], leaves[3], groups)
        return torch.autograd.grad([out, routes.loss], leaves, [dout, torch.ones_like(routes.loss)])
    values = (x, logits, down, up)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        leaves = [t.clone().requires_grad_() for t in values]
        for _ in range(2):
            step(leaves)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        held = step(leaves)
    for replay in range(3):
        new = _trainer(65 + replay)
        fresh = [new[i][:64] if i < 3 else new[i] for i in (0, 1, 3, 4)]
        with torch.no_grad():
            for leaf, value in zip(leaves, fresh):
                leaf.copy_(value)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = step([t.clone().requires_grad_() for t in fresh])
        assert all(torch.equal(a, b) for a, b in zip(held, want)), f"replay {replay}"


def test_streams_and_threads():
    """Steps on two streams at once, and from two threads, are the serial ones."""
    sets = [_server(700), _server(2500)]
    want = [[t.clone() for t in _serve(*s)] for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        got = []
        for s, stream in zip(sets, streams):
            with torch.cuda.stream(stream):
                got.append([_serve(*s) for _ in range(3)])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for runs, w in zip(got, want) for run in runs for a, b in zip(run, w))
    results = [None, None]

    def work(i):
        with torch.cuda.stream(streams[i]):
            results[i] = [_serve(*sets[i]) for _ in range(20)]
            streams[i].synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert all(torch.equal(a, b) for runs, w in zip(results, want) for run in runs for a, b in zip(run, w))


def test_explicit_stream():
    """The `stream` argument: work goes there, not to torch's current stream."""
    stream = torch.cuda.Stream()
    x, logits, _, down, up, ids, scales = _server(300)
    torch.cuda.synchronize()
    routes = H.route_tokens(logits, 2, stream=stream)
    groups = H.group_tokens(routes.experts, 8, stream=stream.cuda_stream)
    rows = H.dispatch_rows(x, groups.rows, groups.ends, stream=stream)
    out = H.combine_rows(rows, groups.rows, routes.weights, stream=stream)
    plan = H.group_tokens(ids, 5, stream=stream)
    adapted, h = H.adapt_rows(x, down, up, plan.ends, plan.slots, scales=scales, hidden=True, stream=stream)
    grad = H.adapter_gradient(h, x, plan.ends, plan.slots, stream=stream)
    dy, dw = H.combine_rows_gradient(out, rows, groups.rows, groups.ends, routes.weights, stream=stream)
    dl = H.route_tokens_gradient(logits, routes, dw, stream=stream)
    stream.synchronize()
    again = H.route_tokens(logits, 2)
    assert torch.equal(routes.weights, again.weights) and torch.equal(dl, H.route_tokens_gradient(logits, again, dw))
    assert torch.equal(out, H.combine_rows(rows, groups.rows, again.weights))
    want, h2 = H.adapt_rows(x, down, up, plan.ends, plan.slots, scales=scales, hidden=True)
    assert torch.equal(adapted, want) and torch.equal(grad, H.adapter_gradient(h2, x, plan.ends, plan.slots))
    assert torch.equal(dy, H.combine_rows_gradient(out, rows, groups.rows, groups.ends, routes.weights)[0])


@pytest.mark.parametrize("module", ["experts", "adapters"])
def test_commands_run(module):
    import subprocess
    import sys
    from pathlib import Path
    res = subprocess.run([sys.executable, "-m", f"paper_2412_08832_amd.{module}"], capture_output=True, text=True,
                         timeout=100, cwd=Path(__file__).resolve().parent.parent)
    assert res.returncode == 0 and "relative error" in res.stdout, res.stdout + res.stderr[-2000:]


@pytest.mark.parametrize("as_number", [False, True])
def test_workspace_of_another_stream(monkeypatch, as_number):
    """A workspace of torch's current stream for work on another one is marked as used there, so that
    it is not handed out again before that work is done."""
    class Spy:
        def __init__(self, tensor):
            self.tensor, self.data_ptr = tensor, tensor.data_ptr

        def record_stream(self, stream):
            marked.append((self.tensor.numel() * 4, stream.cuda_stream))
            self.tensor.record_stream(stream)
    stream, marked, words = torch.cuda.Stream(), [], H._words
    nbytes = H.hadacore_route_workspace_size(20000, 256)
    monkeypatch.setattr(H, "_words", lambda n, *a: Spy(words(n, *a)) if n * 4 == nbytes else words(n, *a))
    logits = torch.randn((20000, 256), device="cuda")
    torch.cuda.synchronize()
    H.route_tokens(logits, 4, stream=stream.cuda_stream if as_number else stream)
    assert marked == [(nbytes, stream.cuda_stream)]
    H.route_tokens(logits, 4, stream=0)
    assert marked[1:] == [(nbytes, torch.cuda.default_stream().cuda_stream)]
    H.route_tokens(logits, 4)
    torch.cuda.synchronize()
    assert len(marked) == 2


def test_offsets_past_32_bits():
    """Rows 2^26 values apart: 40 of them reach past 2^32 bytes, in every operator."""
    m, pitch, width = 40, 1 << 26, 264
    gen = torch.Generator(device="cuda").manual_seed(0)
    room = torch.empty(m * pitch, dtype=torch.float16, device="cuda")
    far = room.view(m, pitch)[:, :width]
    near = torch.randn((m, width), generator=gen, device="cuda").half()
    far.copy_(near)
    groups = H.group_tokens(torch.randint(0, 3, (m,), generator=gen, device="cuda").int(), 3)
    w = torch.rand(m, generator=gen, device="cuda")
    assert torch.equal(H.dispatch_rows(far, groups.rows, groups.ends), H.dispatch_rows(near, groups.rows, groups.ends))
    assert torch.equal(H.combine_rows(far, groups.rows, w), H.combine_rows(near, groups.rows, w))
    dout = torch.randn((m, width), generator=gen, device="cuda").half()
    for a, b in zip(H.combine_rows_gradient(far, dout, groups.rows, groups.ends, w),
                    H.combine_rows_gradient(near, dout, groups.rows, groups.ends, w)):
        assert torch.equal(a, b)
    down, up = (0.1 * torch.randn((3, 20, width), generator=gen, device="cuda")).half(), \
        torch.randn((3, 20, 200), generator=gen, device="cuda").half()
    got, h = H.adapt_rows(far, down, up, groups.ends, groups.slots, hidden=True)
    want, _ = H.adapt_rows(near, down, up, groups.ends, groups.slots, hidden=True)
    assert torch.equal(got, want)
    assert torch.equal(H.adapter_gradient(h, far, groups.ends, groups.slots),
                       H.adapter_gradient(h, near, groups.ends, groups.slots))
    y = torch.randn((m, 200), generator=gen, device="cuda").half()
    want = H.adapt_rows(near, down, up, groups.ends, groups.slots, y=y)
    out = room.view(m, pitch)[:, 512:712]
    out.copy_(y)
    H.adapt_rows(near, down, up, groups.ends, groups.slots, y=out, out=out)
    assert torch.equal(out, want)
    for target, call in ((room.view(m, pitch)[:, 1024 : 1024 + width], lambda o: H.dispatch_rows(near, groups.rows, groups.ends, out=o)),
                         (room.view(m, pitch)[:, 2048 : 2048 + width], lambda o: H.combine_rows(near, groups.rows, w, out=o))):
        assert torch.equal(call(target), call(None))
    logits = room.view(torch.float32).view(m, pitch // 2)[:, 4096 : 4096 + 50]
    logits.copy_(torch.randn((m, 50), generator=gen, device="cuda"))
    close = logits.contiguous()
    routes, want = H.route_tokens(logits, 3), H.route_tokens(close, 3)
    assert all(torch.equal(a, b) for a, b in zip(routes[:5], want[:5]))
    back = room.view(torch.float32).view(m, pitch // 2)[:, 8192 : 8192 + 50]
    want = H.route_tokens_gradient(close, routes, routes.weights)
    assert torch.equal(H.route_tokens_gradient(logits, routes, routes.weights), want)
    assert torch.equal(H.route_tokens_gradient(close, routes, routes.weights, out=back), want)
