"""The training operators under torch's automatic differentiation: a tensor that
requires a gradient gets the operator's own, and nothing is cut off in silence."""
import pytest
import torch

from paper_2608_08340_gb300.train import (distill_loss, embed_lookup, embed_lookup_grad,
                                          embed_pool_grad, embed_pool_train)

from test_gpu_train import DT, _rand, _teacher, _zipf_ids

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(), (7,), (40, 130)])
def test_lookup(dtype, shape):
    table = _rand((500, 64), dtype, 1).requires_grad_()
    ids = torch.full((), 3, device="cuda") if shape == () else _zipf_ids(shape, 500, 2)
    rows = embed_lookup(table, ids, 2.5, torch.float32)
    plain = embed_lookup(table.detach(), ids, 2.5, torch.float32)
    assert rows.requires_grad and not plain.requires_grad and torch.equal(rows, plain)
    grad = _rand((*shape, 64), "f32", 3)
    rows.backward(grad)
    want = embed_lookup_grad(grad.view(-1, 64), ids.reshape(-1), 500, 2.5, DT[dtype])
    assert table.grad.dtype == DT[dtype] and torch.equal(table.grad, want)
    with torch.no_grad():
        assert not embed_lookup(table, ids).requires_grad


def test_lookup_into_a_given_tensor():
    table, ids = _rand((50, 16), "f32", 4).requires_grad_(), torch.tensor([4, -1, 4], device="cuda")
    out = torch.empty(3, 16, device="cuda")
    got = embed_lookup(table, ids, 1.0, out=out)
    assert got.data_ptr() == out.data_ptr() and got.requires_grad
    got.sum().backward()                          # (a broadcast gradient)
    assert (table.grad[4] == 2).all() and table.grad.sum() == 32


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
def test_tail(dtype, out):
    hidden = _rand((9, 50, 72), dtype, 5).requires_grad_()
    mask = torch.arange(50, device="cuda") < torch.arange(0, 45, 5, device="cuda")[:, None]
    query, mean = embed_pool_train(hidden, mask, DT[out])
    assert query.requires_grad and not mean.requires_grad
    grad = _rand((9, 72), out, 6)
    query.backward(grad)
    assert torch.equal(hidden.grad, embed_pool_grad(grad, mean, mask, DT[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("grad", [True, False])
def test_distillation(dtype, grad):
    """The loss is not weighted: its gradient is the upstream one's."""
    logits = _rand((20, 3001), dtype, 7).requires_grad_()
    ids, scores = _teacher(20, 3001, 9, 8)
    weight = torch.rand(20, device="cuda")
    loss, dz = distill_loss(logits, ids, scores, 0.3, weight, grad=grad)
    plain_loss, plain = distill_loss(logits.detach(), ids, scores, 0.3, weight)
    assert loss.requires_grad and torch.equal(loss, plain_loss)
    if grad:
        assert not dz.requires_grad and torch.equal(dz, plain)
    (loss * weight).sum().backward()
    assert torch.equal(logits.grad, plain)


def test_distillation_over_its_scores():
    """Scores that their gradient overwrote have none to give."""
    start = _rand((4, 100), "f32", 9).requires_grad_()
    ids, scores = _teacher(4, 100, 5, 10)
    for out in (lambda z: z, lambda z: z.detach()):
        logits = start * 2
        want = distill_loss(logits.detach().clone(), ids, scores, 0.3)
        loss, dz = distill_loss(logits, ids, scores, 0.3, out=out(logits))
        assert torch.equal(loss, want[0]) and torch.equal(dz, want[1])
        with pytest.raises(RuntimeError, match="inplace"):
            loss.sum().backward()
    apart = torch.empty_like(start)
    loss, dz = distill_loss(start, ids, scores, 0.3, out=apart)
    loss.sum().backward()
    assert dz is apart and torch.equal(start.grad, dz)


@pytest.mark.parametrize("other", [False, True])
def test_a_step_from_the_loss_to_the_table(other):
    """Against the same step in 64 bits."""
    s = torch.cuda.Stream() if other else None
    table, E = _rand((60, 64), "f32", 11).requires_grad_(), _rand((3000, 64), "f32", 12)
    ids = _zipf_ids((8, 30), 60, 13)
    t_ids, t_scores = _teacher(8, 3000, 9, 14)
    torch.cuda.synchronize()
    with torch.cuda.stream(s if other else torch.cuda.current_stream()):
        query, _ = embed_pool_train(embed_lookup(table, ids, 3.0, stream=s), ids >= 0, torch.float32,
                                    stream=s)
        loss, _ = distill_loss(query @ E.T, t_ids, t_scores, 0.2, grad=False, stream=s)
        loss.mean().backward()
    torch.cuda.synchronize()
    t64 = table.detach().double().requires_grad_()
    real = (ids >= 0).double()[:, :, None]
    q64 = torch.nn.functional.normalize((3.0 * t64[ids.clamp(min=0)] * real).sum(1), dim=1)
    log_t = torch.log_softmax(t_scores.double() / 0.2, 1)
    log_p = torch.log_softmax(q64 @ E.double().T / 0.2, 1).gather(1, t_ids)
    (log_t.exp() * (log_t - log_p)).sum(1).mean().backward()
    # fp32 products of 64 terms, held to smoke()'s bound of the same chain
    assert (table.grad.double() - t64.grad).norm() < 1e-4 * t64.grad.norm()


def test_second_derivatives_are_refused():
    table = _rand((50, 16), "f32", 15).requires_grad_()
    rows = embed_lookup(table, torch.tensor([4, 5], device="cuda"))
    g, = torch.autograd.grad((rows * rows).sum(), table, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()
