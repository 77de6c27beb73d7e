"""GPU parity of the training operators on the plans that large calls take: rows that
clusters of every size share, sorts of many tiles, several column slabs, long rows.
References and error bounds are those of test_gpu_train.py."""
import math

import pytest
import torch

from paper_2608_08340_gb300.train import (distill_loss, embed_lookup, embed_lookup_grad,
                                          embed_pool_grad, embed_pool_train)

from test_gpu_train import (DT, U, _check_distill, _distill_plain, _pool_grad_plain, _rand,
                            _tail_mask, _teacher, _within, _zipf_ids)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------- distillation

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kb,q", [(100, 700), (300, 400), (700, 200), (1000, 120), (1100, 120)])
def test_distill_of_many_rows_that_clusters_share(dtype, kb, q):
    """Rows of 2, 4, 8, 16 and 16 larger CTAs, more of them than run at a time, so that
    CTAs of a cluster begin at different moments: the same bits every time, and the
    reference's values."""
    n = kb * 1000 // (2 if dtype == "bf16" else 4) + 5
    logits = _rand((q, n), dtype, kb, 0.2)
    ids, scores = _teacher(q, n, 20, kb + 1)
    loss, dz = distill_loss(logits, ids, scores, 0.1)
    for _ in range(8):
        again, dz2 = distill_loss(logits, ids, scores, 0.1)
        assert torch.equal(again, loss) and torch.equal(dz2, dz)
    for i in (0, q // 2, q - 1):
        part = slice(i, i + 1)
        want, grad, loss_bound, grad_bound = _distill_plain(logits[part], ids[part], scores[part],
                                                            0.1, None)
        _within(loss[part].cpu(), want, loss_bound, "f32", f"loss {i}")
        _within(dz[part].cpu(), grad, grad_bound, dtype, f"gradient {i}")


# ------------------------------------------------------- the embedding tail

@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("d", [8, 392, 4104])
@pytest.mark.parametrize("size,by", [(1e25, 1.0), (2e37, 1.0), (1e-25, 1.0), (1e-36, 1e-3),
                                     (1e-41, 1e-9)])
def test_pool_grad_of_means_whose_squares_leave_the_range(dtype, out, d, size, by):
    """Finite means of any size have the definition's gradient."""
    mask = _tail_mask(6, 9, d)
    mean, grad = _rand((6, d), "f32", d, 1.0), _rand((6, d), dtype, d + 1, by)
    mean[0] *= size
    mean[3] *= size
    mean[4] *= size
    mean[4, 1:] = 0                               # one value alone
    mean[5, ::2] *= size                          # large and small ones
    row, bound = _pool_grad_plain(grad, mean, mask)
    _within(embed_pool_grad(grad, mean, mask, DT[out], per_token=False).cpu(), row, bound, out)


def test_pool_grad_of_an_infinite_mean_is_not_a_number():
    mask = torch.ones(4, 6, dtype=torch.bool, device="cuda")
    mask[:, 4:] = False
    mean, grad = _rand((4, 64), "f32", 1), _rand((4, 64), "f32", 2)
    clean = embed_pool_grad(grad, mean, mask, torch.float32)
    mean[1, 3], mean[2, 5] = math.inf, -math.inf
    got = embed_pool_grad(grad, mean, mask, torch.float32)
    assert got[1:3, :4].isnan().all() and (got[1:3, 4:] == 0).all()
    assert torch.equal(got[[0, 3]], clean[[0, 3]])


# ------------------------------------------------------------------ streams

def _calls():
    """(call of a stream and an output or None, its inputs) for every operator."""
    table, ids = _rand((3000, 512), "f32", 1), torch.randint(0, 3000, (64, 90), device="cuda")
    hidden, mask = _rand((64, 90, 512), "f32", 2), torch.ones(64, 90, dtype=torch.bool, device="cuda")
    mean, grad = _rand((64, 512), "f32", 3), _rand((64, 512), "f32", 4)
    logits, weight = _rand((64, 5000), "f32", 5), torch.rand(64, device="cuda")
    t_ids, t_scores = _teacher(64, 5000, 9, 6)
    return {
        "lookup": (lambda a, s: embed_lookup(*a, stream=s), [table, ids]),
        "lookup_grad": (lambda a, s: embed_lookup_grad(*a, 3000, stream=s), [hidden, ids]),
        "pool_train": (lambda a, s: embed_pool_train(*a, stream=s), [hidden, mask]),
        "pool_grad": (lambda a, s: embed_pool_grad(*a, stream=s), [grad, mean, mask]),
        "distill": (lambda a, s: distill_loss(*a[:3], 0.3, a[3], stream=s),
                    [logits, t_ids, t_scores, weight]),
    }


@pytest.mark.parametrize("name", ["lookup", "lookup_grad", "pool_train", "pool_grad", "distill"])
def test_inputs_may_be_dropped_behind_a_call_on_another_stream(name):
    """The memory of a dropped input is not given away while the stream that the call
    was given still has to read it."""
    call, inputs = _calls()[name]
    want = call(inputs, None)
    s = torch.cuda.Stream()
    mine = [t.clone() for t in inputs]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)            # cycles: about a tenth of a second
    got = call(mine, s)
    del mine
    others = [torch.zeros_like(t) for t in inputs for _ in range(3)]     # on the current stream
    torch.cuda.current_stream().synchronize()
    s.synchronize()
    for a, b in zip(want if isinstance(want, tuple) else [want],
                    got if isinstance(got, tuple) else [got]):
        assert torch.equal(a, b)
    del others


# ------------------------------------------------- outputs beside the inputs

def test_outputs_between_the_rows_of_the_inputs():
    """Rows that lie between the other's rows are apart from them; over them, refused."""
    both = _rand((40, 2048), "f32", 1)
    logits, other = both[:, :1000], both[:, 1000:2000]
    ids, scores = _teacher(40, 1000, 9, 2)
    want_loss, want = distill_loss(logits.clone(), ids, scores, 0.3)
    loss, dz = distill_loss(logits, ids, scores, 0.3, out=other)
    assert dz is other and torch.equal(dz, want) and torch.equal(loss, want_loss)
    for out in (both[:, 999:1999], both[:, 1:1001], both.view(-1)[:40 * 1000].view(40, 1000)):
        with pytest.raises(RuntimeError, match="overlap"):
            distill_loss(logits, ids, scores, 0.3, out=out)
    wide = _rand((50, 96), "f32", 3)
    rows = torch.tensor([3, 49, 0], device="cuda")
    want = embed_lookup(wide[:, :32], rows, 2.0)
    out = wide[7, 32:].view(2, 32)                # in a gap of the table
    assert torch.equal(embed_lookup(wide[:, :32], rows[:2], 2.0, out=out), want[:2])
    with pytest.raises(RuntimeError, match="overlap"):
        embed_lookup(wide[:, :32], rows, 2.0, out=wide[7].view(3, 32))
    grad = _rand((6, 5, 32), "f32", 4)
    ids = torch.randint(0, 10, (6, 5), device="cuda")
    want = embed_lookup_grad(grad[2:].clone(), ids[2:], 10)
    assert torch.equal(embed_lookup_grad(grad[2:], ids[2:], 10, out=grad[:2].view(10, 32)), want)
    with pytest.raises(RuntimeError, match="overlap"):
        embed_lookup_grad(grad[1:], ids[1:], 10, out=grad[:2].view(10, 32))


# ------------------------------------------------------- gradient of the lookup

def _check_grad(grad, ids, vocab, scale, out):
    """Against sums in 64 bits, formed on the GPU for some columns at a time; the bound
    is that of test_gpu_train.py."""
    got = embed_lookup_grad(grad, ids, vocab, scale, DT[out])
    flat = ids.reshape(-1).long()
    real = (flat >= 0) & (flat < vocab)
    at = flat[real]
    count = torch.bincount(at, minlength=vocab)[:, None]
    for lo in range(0, grad.shape[-1], 256):
        g = grad[..., lo:lo + 256].reshape(flat.numel(), -1)[real].double()
        zero = torch.zeros(vocab, g.shape[1], dtype=torch.float64, device="cuda")
        exact = torch.index_add(zero, 0, at, g) * scale
        mag = torch.index_add(zero, 0, at, g.abs()) * abs(scale)
        _within(got[:, lo:lo + 256], exact, (count + 1) * U * mag, out, f"columns from {lo}")


def _check_whole_numbers(shape, dtype, ids, vocab):
    """Sums of small whole numbers are exact in fp32 (below 2^24) in any order: no token is
    lost, counted twice or added to another row."""
    assert 3 * ids.numel() < 2 ** 24
    g = torch.Generator(device="cuda").manual_seed(vocab)
    grad = torch.randint(-3, 4, shape, generator=g, device="cuda").to(DT[dtype])
    flat = ids.reshape(-1).long()
    real = (flat >= 0) & (flat < vocab)
    want = torch.zeros(vocab, shape[-1], dtype=torch.float64, device="cuda")
    for lo in range(0, shape[-1], 256):
        part = grad[..., lo:lo + 256].reshape(flat.numel(), -1)[real].double()
        want[:, lo:lo + 256].index_add_(0, flat[real], part)
    assert torch.equal(embed_lookup_grad(grad, ids, vocab).double(), want)


# Row widths of every number of groups a lane, and of several column slabs; from 69632
# tokens x slabs on, units of more than 16 items, up to 64 and 128.
@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("vocab,dim,shape", [
    (3000, 264, (50, 100)), (3000, 384, (50, 100)), (3000, 392, (50, 100)), (3000, 520, (50, 100)),
    (3000, 768, (50, 100)), (3000, 776, (50, 100)), (3000, 1024, (7, 801)), (2000, 1032, (50, 100)),
    (700, 4104, (60, 100)), (9, 2056, (5, 600)), (2000, 520, (100, 801)), (30522, 1032, (100, 400)),
    (500, 768, (300, 999)), (50, 128, (40, 7001)), (500, 4104, (150, 401)), (3000, 8192, (90, 301))])
def test_lookup_grad_of_wide_rows_and_large_units(dtype, out, vocab, dim, shape):
    ids = _zipf_ids(shape, vocab, dim + vocab)
    _check_grad(_rand((*shape, dim), dtype, dim), ids, vocab, 0.7, out)
    _check_whole_numbers((*shape, dim), dtype, ids, vocab)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,tokens", [(768, 3000), (768, 300000), (1032, 100000), (4104, 70000)])
def test_lookup_grad_of_a_few_long_rows(dtype, dim, tokens):
    """Rows that cross many units, that end where a unit does, and single tokens beside them."""
    ids = torch.full((tokens,), 40, device="cuda")
    ids[tokens // 3:] = 41
    ids[tokens // 2:] = 90
    ids[::1000] = torch.arange(0, (tokens + 999) // 1000, device="cuda") % 97
    grad = _rand((tokens, dim), dtype, dim)
    _check_grad(grad, ids, 100, 1.0, "f32")
    _check_whole_numbers((tokens, dim), dtype, ids, 100)
    _check_grad(grad, torch.arange(tokens, device="cuda") // 256, tokens // 256 + 1, 1.0, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,texts,tokens", [(768, 1000, 300), (64, 1000, 300), (1032, 200, 250)])
def test_lookup_grad_of_many_texts_that_share_a_gradient(dtype, dim, texts, tokens):
    rows = _rand((texts, 1, dim), dtype, dim)
    _check_grad(rows.expand(-1, tokens, -1), _zipf_ids((texts, tokens), 30522, 1), 30522, 3.0, "f32")


# Tiles of 1024 tokens to 32768 of them, of 4096 beyond; more than 128 tiles beyond
# 524288; one, two and three passes over the ids' digits.
@pytest.mark.parametrize("bits", [torch.int32, torch.int64])
@pytest.mark.parametrize("vocab", [5, 600, 2 ** 18, 2 ** 18 + 1, 1000003])
@pytest.mark.parametrize("tokens", [2049, 32768, 32769, 44800, 131072, 131073, 524288, 524289, 1200001])
def test_lookup_grad_of_sorts_of_every_size(bits, vocab, tokens):
    if vocab < 2000:
        ids = _zipf_ids((tokens,), vocab, tokens)
    else:                                         # all of the digits
        ids = torch.randint(-vocab // 8, vocab + vocab // 8, (tokens,), device="cuda",
                            generator=torch.Generator(device="cuda").manual_seed(tokens))
        ids[::3] = vocab - 1 - ids[::3] % 50
    _check_grad(_rand((tokens, 8), "f32", vocab), ids.to(bits), vocab, 1.0, "f32")
    _check_whole_numbers((tokens, 8), "bf16", ids.to(bits), vocab)


# ------------------------------------------- distillation of more than 1 MB a row

@pytest.mark.parametrize("dtype,n", [("bf16", 600007), ("f32", 300011), ("bf16", 1048576)])
@pytest.mark.parametrize("k", [129, 200, 256])
def test_distill_of_many_results_in_large_rows(dtype, n, k):
    q = 6
    logits = _rand((q, n), dtype, n, 0.3)
    ids, scores = _teacher(q, n, k, k)
    ids[0, ::3] = ids[0, 1]                       # repeated ones
    ids[1, k // 2:] = ids[1, :k - k // 2].clone()
    logits[2, ids[2, :50]] = -math.inf            # hidden ones
    logits[3, n // 4:n // 2] = torch.finfo(logits.dtype).min
    ids[4, 7:] = -1                               # few
    scores[5, k - 100:] = -math.inf
    ids[5, 0], ids[5, 1] = n - 1, 0
    weight = torch.linspace(-1, 2, q, device="cuda")
    _, dz = _check_distill(logits, ids, scores, 0.2, weight)
    assert (dz[2, ids[2, :50]] == 0).all() and (dz[3, n // 4:n // 2] == 0).all()
