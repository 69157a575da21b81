"""The MLP operators where offsets pass 32 bits: results of more than 2^31 elements, and experts behind the first 4 GiB of weights."""
import pytest
import torch

from paper_2608_24070_amd import slim

pytestmark = pytest.mark.gpu


def test_gradient_over_more_than_2_31_elements():
    m, k = 40000, 56001
    dh = torch.full((m, k), 0.5, dtype=torch.bfloat16, device="cuda")
    u = torch.zeros((m, k), dtype=torch.bfloat16, device="cuda")
    last = torch.randn((64, k), device="cuda").bfloat16()
    u[-64:] = last
    du, _, db = slim.act_bwd(dh, u, act="silu", bias=True)
    want, _, _ = slim.act_bwd(dh[-64:], last, act="silu")
    assert torch.equal(du[-64:], want) and bool((du[:-64] == 0.25).all())
    # a quarter from each of the other rows, exact in fp32, and the last rows' as 64 bits have them
    s = torch.sigmoid(last.double())
    ref = 0.25 * (m - 64) + (0.5 * (s + last.double() * s * (1 - s))).sum(0)
    assert bool(((db.double() - ref).abs() <= 2.0 ** -20 * ref).all())


def test_product_of_more_than_2_31_elements():
    m, n, k = 70001, 32768, 128
    x = torch.randint(-2, 3, (m, k), device="cuda").bfloat16()
    w = torch.randint(-2, 3, (n, k), device="cuda").float()
    p = slim.pack8(w)
    y = slim.linear8_act(x, p, act="relu")
    for rows in (slice(0, 100), slice(65400, 65700), slice(m - 100, m)):
        assert torch.equal(y[rows].float(), torch.relu(x[rows].float() @ w.t()))
    del y
    q = slim.linear8_act(x, p, act="relu", q8=True)
    at = torch.tensor([0, 65535, m - 1], device="cuda")
    rows = {"codes": q["codes"][at], "exps": q["exps"][at], "M": 3, "K": n}
    assert torch.equal(slim.dequant8(rows, torch.float32), slim.dequant8(slim.quant8(torch.relu(x[at].float() @ w.t())), torch.float32))


@pytest.mark.parametrize("m", [1, 9])
def test_experts_behind_the_first_4_gib(m):
    e, d, f = 150, 4096, 8192
    gen = torch.Generator("cuda").manual_seed(m)
    few = {"gate": torch.randn((2, f, d), generator=gen, device="cuda") / 64, "down": torch.randn((2, d, f), generator=gen, device="cuda") / 90}
    small, big = {}, {}
    for name, w in few.items():
        s = small[name] = slim.pack8_experts(w)
        b = big[name] = {"codes": torch.empty((e,) + s["codes"].shape[1:], dtype=torch.uint8, device="cuda"),
                         "exps": torch.empty((e,) + s["exps"].shape[1:], dtype=torch.uint8, device="cuda"), "E": e, "N": s["N"], "K": s["K"]}
        for part in ("codes", "exps"):
            b[part][3], b[part][e - 1] = s[part][0], s[part][1]
    x = torch.randn((m, d), generator=gen, device="cuda").bfloat16()
    ids = torch.randint(0, 2, (m, 1), generator=gen, device="cuda", dtype=torch.int32)
    ids[0] = 1
    weights = torch.rand((m, 1), generator=gen, device="cuda")
    want = slim.moe8(x, small["gate"], None, small["down"], ids, weights)
    far = torch.where(ids == 1, e - 1, 3).int()
    got = slim.moe8(x, big["gate"], None, big["down"], far, weights)
    assert bool(want.isfinite().all()) and bool(want.any())
    # the parts that the reduction is cut in may go by the number of experts
    assert bool(((got.double() - want.double()).norm() / want.double().norm()) < 2.0 ** -8)
