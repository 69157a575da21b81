"""Results of the MLP operators in the places that they may take: an operand's very rows, and beside operands in one buffer. The same
bits as in a place of their own."""
import pytest
import torch

from paper_2608_24070_amd import slim

pytestmark = pytest.mark.gpu

BF16 = slim.SLIM_BF16
# few rows (quantised in the launch, from codes), tiles, 64-column tiles and slices by sums in memory
SIZES = [(3, 200, 300), (40, 333, 600), (300, 333, 600), (1500, 2050, 300), (64, 515, 28672)]


def rand(*s):
    return torch.randn(s, device="cuda").bfloat16()


def workspace(n):
    return torch.full((n + 16,), 0xFF, dtype=torch.uint8, device="cuda")


def checked(status):
    assert status == slim.SLIM_OK, slim.SlimError(status, "call")


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
def test_forward(m, n, k, act):
    print(f"linear8_act in place m={m} n={n} k={k} {act}", flush=True)
    x, w = rand(m, k), torch.randn((n, k), device="cuda") * k ** -0.5
    p, mul, res = slim.pack8(w), rand(m, n), rand(m, n)
    y, z = slim.linear8_act(x, p, act=act, mul=mul, residual=res, pre=True)
    ws = workspace(slim.slim_linear8_act_workspace(BF16, m, n, k, BF16, 0))

    def call(mt, rt, yt, zt):
        checked(slim.slim_linear8_act(x.data_ptr(), BF16, None, m, n, k, k, p["codes"].data_ptr(), p["exps"].data_ptr(), slim.ACTS[act], None,
                                      slim.SLIM_F32, mt.data_ptr(), mt.stride(0), rt.data_ptr(), rt.stride(0), BF16, 0, yt.data_ptr(), yt.stride(0),
                                      None, zt.data_ptr(), zt.stride(0), None, ws.data_ptr(), ws.numel(), slim._stream_on(0)))
        assert torch.equal(yt, y) and torch.equal(zt, z)

    for cross in (False, True):            # Y and pre each in the place of one of the two
        a, b = mul.clone(), res.clone()
        call(a, b, *((b, a) if cross else (a, b)))
    # one buffer: factor, residual, result and argument side by side, and the result in the factor's columns
    wide = torch.full((m, 4 * n + 5), -7.0, dtype=torch.bfloat16, device="cuda")
    part = [wide[:, i * n + i:(i + 1) * n + i] for i in range(4)]
    part[0].copy_(mul)
    part[1].copy_(res)
    call(*part)
    assert torch.equal(part[0], mul) and torch.equal(part[1], res) and bool((wide[:, n::n + 1][:, :4] == -7).all())
    call(part[0], part[1], part[0], part[3])
    # a buffer's rows in turn
    if m > 1:
        tall = torch.zeros((2 * m, n), dtype=torch.bfloat16, device="cuda")
        mt, yt = tall[0::2], tall[1::2]
        mt.copy_(mul)
        call(mt, res, yt, torch.empty_like(z))
    # one row has no stride
    if m > 2:
        one = slim.linear8_act(x[:1], p, act=act, mul=mul[:1], residual=res[:1])
        row = mul[:1].clone()
        wide_row = torch.as_strided(row, (1, n), (n + 9, 1))
        assert torch.equal(slim.linear8_act(x[:1], p, act=act, mul=row, residual=res[:1], out=wide_row), one)


@pytest.mark.parametrize("m,n,k", SIZES + [(1, 130, 4100), (100, 129, 4097)])
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
def test_backward(m, n, k, act):
    # n: the reduction, k: the columns of dh
    n, k = k, n
    print(f"gradients in place m={m} n={n} k={k} {act}", flush=True)
    dy, w = rand(m, n), torch.randn((n, k), device="cuda") * n ** -0.5
    p, u, mul, dh = slim.pack8(w, bwd=True), rand(m, k), rand(m, k), rand(m, k)
    a = slim.ACTS[act]
    ws = workspace(max(slim.slim_bwd_dx8_act_workspace(BF16, m, n, k, BF16, 1), slim.slim_act_bwd_workspace(m, k, 1)))

    def product(src, ut, mt, dut, dmt):
        db = torch.empty(k, dtype=torch.bfloat16, device="cuda")
        checked(slim.slim_bwd_dx8_act(src.data_ptr(), BF16, None, m, n, k, src.stride(0), p["codesT"].data_ptr(), p["expsT"].data_ptr(), a,
                                      ut.data_ptr(), BF16, None, ut.stride(0), mt.data_ptr(), None, mt.stride(0), BF16, dut.data_ptr(), dut.stride(0),
                                      dmt.data_ptr(), dmt.stride(0), db.data_ptr(), ws.data_ptr(), ws.numel(), slim._stream_on(0)))
        return dut, dmt, db

    def alone(src, ut, mt, dut, dmt):
        db = torch.empty(k, device="cuda")
        checked(slim.slim_act_bwd(src.data_ptr(), BF16, src.stride(0), m, k, a, ut.data_ptr(), BF16, None, ut.stride(0), mt.data_ptr(), None,
                                  mt.stride(0), dut.data_ptr(), dut.stride(0), dmt.data_ptr(), dmt.stride(0), db.data_ptr(), ws.data_ptr(), ws.numel(),
                                  slim._stream_on(0)))
        return dut, dmt, db

    for call, src in ((product, dy), (alone, dh)):
        want = [t.clone() for t in call(src, u, mul, torch.empty_like(u), torch.empty_like(u))]
        same = lambda got: all(torch.equal(s, t) for s, t in zip(got, want))
        for cross in (False, True):
            ut, mt = u.clone(), mul.clone()
            assert same(call(src, ut, mt, *((mt, ut) if cross else (ut, mt))))
        # side by side in one buffer, and the gradient in u's columns
        wide = torch.full((m, 4 * k + 5), -7.0, dtype=torch.bfloat16, device="cuda")
        part = [wide[:, i * k + i:(i + 1) * k + i] for i in range(4)]
        part[0].copy_(u)
        part[1].copy_(mul)
        assert same(call(src, *part)) and torch.equal(part[0], u) and torch.equal(part[1], mul)
        assert same(call(src, part[0], part[1], part[0], part[3]))
        if call is alone:
            for cross in (False, True):
                s, other = dh.clone(), torch.empty_like(dh)
                assert same(call(s, u, mul, *((other, s) if cross else (s, other))))
    # a 16-bit dY's own rows: it is read before anything is written
    if m * n >= m * k and m > 1:
        want = [t.clone() for t in product(dy, u, mul, torch.empty_like(u), torch.empty_like(u))]
        s = dy.clone()
        got = product(s, u, mul, s.view(-1)[:m * k].view(m, k), torch.empty_like(u))
        assert all(torch.equal(x, y) for x, y in zip(got, want))


# one row, few rows, and rows whose reduction is in parts (their sums are added by a launch of its own)
@pytest.mark.parametrize("m,e,d,f,top", [(1, 8, 300, 200, 3), (9, 4, 300, 200, 2), (40, 6, 130, 2100, 4)])
def test_experts(m, e, d, f, top):
    gate, up, down = (slim.pack8_experts(torch.randn((e, *s), device="cuda") * s[1] ** -0.5) for s in ((f, d), (f, d), (d, f)))
    x, res = rand(m, d), rand(m, d)
    ids, weights = slim.route(x, rand(e, d), top)
    want = slim.moe8(x, gate, up, down, ids, weights, residual=res)
    wide = torch.full((m, 3 * d + 4), -7.0, dtype=torch.bfloat16, device="cuda")
    part = [wide[:, i * d + i:(i + 1) * d + i] for i in range(3)]
    part[0].copy_(x)
    part[1].copy_(res)
    assert torch.equal(slim.moe8(part[0], gate, up, down, ids, weights, residual=part[1], out=part[2]), want)
    assert torch.equal(part[0], x) and torch.equal(part[1], res)
    assert torch.equal(slim.moe8(part[0], gate, up, down, ids, weights, residual=part[1], out=part[1]), want)
    part[1].copy_(res)
    assert torch.equal(slim.moe8(part[0], gate, up, down, ids, weights, residual=part[1], out=part[0]), want)
    # X's memory at another stride
    flat = torch.empty(m * (d + 8), dtype=torch.bfloat16, device="cuda")
    xs, out = flat[:m * d].view(m, d), flat.view(m, d + 8)[:, :d]
    xs.copy_(x)
    assert torch.equal(slim.moe8(xs, gate, up, down, ids, weights, residual=res, out=out), want)
