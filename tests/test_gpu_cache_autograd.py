"""The calls around the KV cache under autograd: the rotation's gradient, refusals, tensors written in place."""
import pytest
import torch

import cache_reference as ref
from test_gpu_cache_ops import BF, FP, close_to_rounding, gen, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def paged():
    from paper_2607_27692_b200 import build, paged
    build.build()
    return paged


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("rot,interleaved", [(64, False), (32, True), (10, False)])
def test_the_rotation_is_recorded(paged, dtype, inverse, rot, interleaved):
    """Gradients of q and k against the 64-bit formula's; once through a layer, upstream gradients of any stride."""
    n, d = 9, 64
    rope = paged.Rope(d, rot, interleaved=interleaved, scaling="yarn", factor=4.0, original_len=64)
    w, amp = ref.frequencies(rot, 10000.0, "yarn", 4.0, 64)
    g = gen(501)
    q = torch.randn(n, 4, d, generator=g, device="cuda").to(dtype).requires_grad_()
    k = torch.randn(n, 2, d, generator=g, device="cuda").to(dtype).requires_grad_()
    pos = ints(list(range(300, 300 + n)))
    up_q = torch.randn(n, 4, d, generator=g, device="cuda").to(dtype)
    up_k = torch.randn(n, d, 2, generator=g, device="cuda").to(dtype).transpose(1, 2)       # not contiguous
    want_q, want_k = (ref.rotate(u, pos, w, amp, interleaved, not inverse) for u in (up_q, up_k))
    qo, ko = rope.apply_pair(q, k, pos, inverse=inverse)
    assert qo.requires_grad and ko.requires_grad
    close_to_rounding(qo.detach(), ref.rotate(q.detach(), pos, w, amp, interleaved, inverse), dtype)
    gq, gk = torch.autograd.grad((qo, ko), (q, k), (up_q, up_k))
    close_to_rounding(gq, want_q, dtype)
    close_to_rounding(gk, want_k, dtype)
    # one of the two alone, and a single tensor
    qo, ko = rope.apply_pair(q.detach(), k, pos, inverse=inverse)
    assert torch.equal(torch.autograd.grad(ko, k, up_k)[0], gk)
    qo, none = rope.apply_pair(q, None, pos, inverse=inverse)
    assert none is None and torch.equal(torch.autograd.grad(qo, q, up_q)[0], gq)
    assert torch.equal(torch.autograd.grad(rope.apply(q, pos, inverse=inverse), q, up_q)[0], gq)
    # a gradient without strides (of a sum), into leaves that add up
    rope.apply(q, pos, inverse=inverse).sum().backward()
    close_to_rounding(q.grad, ref.rotate(torch.ones_like(up_q), pos, w, amp, interleaved, not inverse), dtype)
    # the gradient's gradient is the rotation again
    up = up_q.clone().requires_grad_()
    first, = torch.autograd.grad(rope.apply(q, pos, inverse=inverse), q, up, create_graph=True)
    second, = torch.autograd.grad(first, up, up_q)
    assert torch.equal(second, rope.apply(up_q, pos, inverse=inverse))
    # without autograd nothing is recorded, and the numbers are the same
    with torch.no_grad():
        plain = rope.apply(q, pos, inverse=inverse)
    assert not plain.requires_grad and torch.equal(plain, rope.apply(q, pos, inverse=inverse).detach())


def test_the_gradient_is_that_of_differences(paged):
    """Along random directions: the map is linear, so f(x + h) - f(x) = f(h) with no remainder but rounding."""
    n, H, d = 5, 2, 128
    rope = paged.Rope(d, interleaved=True)
    g = gen(511)
    x, h, up = (torch.randn(n, H, d, generator=g, device="cuda").to(FP) for _ in range(3))
    pos = ints([7, 1000, 0, 99999, 12])
    y = x.clone().requires_grad_()
    grad, = torch.autograd.grad(rope.apply(y, pos), y, up)
    lhs = (rope.apply(h, pos).double() * up.double()).sum()
    rhs = (grad.double() * h.double()).sum()
    # each rotated element is rounded once, 2^-11 of it
    bound = 2.0 ** -11 * ((rope.apply(h, pos).double() * up.double()).abs().sum() + (grad.double() * h.double()).abs().sum()) * (1 + 2.0 ** -9)
    assert (lhs - rhs).abs() <= bound


def test_gradients_that_would_be_lost_are_refused(paged):
    d, H, page = 64, 2, 16
    rope = paged.Rope(d)
    x = torch.randn(3, H, d, generator=gen(521), device="cuda").to(BF)
    leaf = x.clone().requires_grad_()
    pos, lens, table = ints([0, 1, 2]), ints([1, 1, 1]), ints([[0], [1], [2]])
    q4, half = paged.KVPages(3, H, page, d, "q4"), paged.KVPages(3, H, page, d, "bf16")
    out, lse = torch.zeros_like(x), torch.zeros(3, H, device="cuda")
    rows = torch.zeros(3, H, 1, d, dtype=BF, device="cuda")
    calls = [
        lambda a: rope.apply(a, pos, out=out), lambda a: rope.apply(x, pos, out=a), lambda a: rope.apply(a, pos, out=a),
        lambda a: rope.apply_pair(x, a, pos, k_out=out), lambda a: rope.apply_pair(x, x, pos, q_out=a),
        lambda a: q4.append(a, x, lens, table), lambda a: half.append(x, a, lens, table),
        lambda a: q4.append(x, x, lens, table, rope=rope, q=a), lambda a: q4.append(x, x, lens, table, rope=rope, q=x, q_out=a),
        lambda a: q4.attend(a, lens, table), lambda a: q4.attend(x, lens, table, out=a),
    ]
    for call in calls:
        with pytest.raises(paged._rt.RetopkError, match="no_grad"):
            call(leaf)
        with torch.no_grad():
            call(leaf)
        call(x.clone())
    with pytest.raises(paged._rt.RetopkError, match="no_grad"):
        q4.gather(rows.clone().requires_grad_(), None, lens, table)
    with pytest.raises(paged._rt.RetopkError, match="no_grad"):
        q4.attend(x, lens, table, lse=lse.clone().requires_grad_())
    with torch.no_grad():
        q4.gather(rows.clone().requires_grad_(), None, lens, table)


def test_a_captured_gradient(paged):
    """Forward and backward passes in one graph replay like the eager ones."""
    n, H, d = 33, 4, 128
    rope = paged.Rope(d)
    x = torch.randn(n, H, d, generator=gen(531), device="cuda").to(BF)
    up = torch.randn(n, H, d, generator=gen(532), device="cuda").to(BF)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    leaf = x.clone().requires_grad_()

    def step():
        return torch.autograd.grad(rope.apply(leaf, pos), leaf, up)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    pos.add_(1000)
    up.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, rope.apply(up, pos, inverse=True))


def test_tensors_written_in_place_are_marked(paged):
    """A tensor that autograd has saved and a call then writes: the backward pass is refused, as after any operator of torch."""
    d, H, page = 64, 2, 16
    rope = paged.Rope(d)
    pos, lens, table = ints([0, 1, 2]), ints([1, 1, 1]), ints([[0], [1], [2]])
    w = torch.ones(1, device="cuda", dtype=BF, requires_grad=True)

    def fresh(*shape, dtype=BF):
        return torch.randn(*(shape or (3, H, d)), generator=gen(541), device="cuda").to(dtype)

    k16, v16 = fresh(3, H, page, d), fresh(3, H, page, d)
    half, q4 = paged.KVPages.wrap(k16, v16), paged.KVPages(3, H, page, d, "q4")
    x = fresh()
    a, b, c, e, f, g, h, lse = (fresh() for _ in range(8))
    rows = [fresh(3, H, 1, d) for _ in "kv"]
    lse = fresh(3, H, dtype=torch.float32)
    writes = [
        ([a], lambda: rope.apply(a, pos, out=a)), ([b], lambda: rope.apply(x, pos, out=b)),
        ([c, e], lambda: rope.apply_pair(x, x, pos, q_out=c, k_out=e)), ([f, k16, v16], lambda: half.append(x, x, lens, table, rope=rope, q=x, q_out=f)),
        ([k16[1:], v16.view(-1)], lambda: half.append(x, x, lens, table)), ([q4.k_scale, q4.v_scale], lambda: q4.append(x, x, lens, table)),
        (rows, lambda: q4.gather(*rows, lens, table)), ([g, lse], lambda: q4.attend(x, lens, table, out=g, lse=lse)),
        ([h], lambda: q4.attend(h, lens, table, out=h)),
    ]
    for tensors, call in writes:
        results = [(t * w.to(t.dtype)).sum() for t in tensors]           # the product saves t
        kept = (x * w).sum()
        before = [t._version for t in tensors]
        call()
        assert all(t._version > n for t, n in zip(tensors, before))
        for r in results:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                r.backward()
        kept.backward()                                                  # inputs are not marked
    codes = [q4.k._version, q4.v._version]
    q4.append(x, x, lens, table)
    assert [q4.k._version, q4.v._version] > codes
    # tensors without a version counter are written all the same
    with torch.inference_mode():
        cache = paged.KVPages(3, H, page, d, "bf16")
        y = fresh()
    cache.append(x, x, lens, table, rope=rope, q=x, q_out=y)
    rope.apply(y, pos, out=y)
    assert torch.equal(cache.v[0, :, 0], x[0])
    # a cache whose tensors require a gradient
    leaf = paged.KVPages.wrap(k16.detach().clone().requires_grad_(), v16.detach().clone())
    with pytest.raises(paged._rt.RetopkError, match="no_grad"):
        leaf.append(x, x, lens, table)
    with pytest.raises(paged._rt.RetopkError, match="no_grad"):
        leaf.gather(*rows, lens, table)
    with torch.no_grad():
        leaf.append(x, x, lens, table)
