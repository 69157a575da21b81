"""The 8-bit path over operands of more than 2^32 elements: rows past that offset are what the same rows give alone."""
import pytest
import torch

from paper_2608_24070_amd import slim

pytestmark = pytest.mark.gpu

M, K, TAIL = 530000, 8192, 300            # 4.34e9 elements


@pytest.fixture(scope="module")
def rows():
    # integers of -2 .. 2 in a tenth of the places: sums over the reduction of 8192 and over the last rows are exact
    gen = torch.Generator("cuda").manual_seed(1)
    X = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    for part in (X[:TAIL], X[-TAIL:]):
        part.copy_(torch.randint(-2, 3, part.shape, generator=gen, device="cuda") * (torch.rand(part.shape, generator=gen, device="cuda") < 0.1))
    yield X
    del X
    torch.cuda.empty_cache()


def ends(t):
    return t[:TAIL], t[-TAIL:]


def test_quant_product_and_gradient(rows):
    print("quant8", flush=True)
    q = slim.quant8(rows)
    for got, x in zip(zip(ends(q["codes"]), ends(q["exps"])), ends(rows)):
        alone = slim.quant8(x)
        assert torch.equal(got[0], alone["codes"]) and torch.equal(got[1], alone["exps"])
    print("linear8", flush=True)
    W = rows[-40:].float()
    p = slim.pack8(W)
    Y = slim.linear8(q, p, dtype=torch.float16)
    for y, x in zip(ends(Y), ends(rows)):
        assert torch.equal(y.float(), (x.double() @ W.double().T).float().half().float())
    assert not bool(Y[TAIL:-TAIL].any())
    print("grad_w8", flush=True)
    dY = torch.ones((M, 24), dtype=torch.bfloat16, device="cuda")
    dY[::2] = -1
    gW = slim.grad_w8(dY, q)
    want = sum(d.double().T @ x.double() for d, x in zip(ends(dY), ends(rows)))
    assert torch.equal(gW.double(), want)
    print("dequant8", flush=True)
    back = slim.dequant8(q, dtype=torch.bfloat16)
    assert all(torch.equal(b, x) for b, x in zip(ends(back), ends(rows)))
    assert not bool(back[M // 2].any())


def test_norm_and_its_gradient(rows):
    g = torch.linspace(0.5, 1.5, K, device="cuda")
    print("norm", flush=True)
    y, mean, rstd = slim.norm(rows, g)
    for got, x in zip(zip(ends(y), ends(mean), ends(rstd)), ends(rows)):
        assert all(torch.equal(a, b) for a, b in zip(got, slim.norm(x, g)))
    print("norm to 8 bits", flush=True)
    q, _, _ = slim.norm(rows, g, q8=True)
    for c, e, x in zip(ends(q["codes"]), ends(q["exps"]), ends(rows)):
        alone = slim.norm(x, g, q8=True)[0]
        assert torch.equal(c, alone["codes"]) and torch.equal(e, alone["exps"])
    print("norm_bwd", flush=True)
    dx, _, _ = slim.norm_bwd(y, rows, g, mean, rstd)
    for got, d, x, mu, rs in zip(ends(dx), ends(y), ends(rows), ends(mean), ends(rstd)):
        assert torch.equal(got, slim.norm_bwd(d, x, g, mu, rs)[0])
