"""slim_norm on rows of one sign, where the roundings of a sum need not cancel, against the oracle in 64 bits.

Bounds, with v = 2^-24. A sum over a row of K rounds once for each value of its longest chain: the 8 V values of a thread (V
vectors of 8), 6 of the wave, and where T > 64 threads share a row the T / 64 waves' one after the other, with one for each of
the two quotients; rows past 32768, and past 16384 where K % 8, take 8 values a vector, ceil(K / 8192) vectors, 6, 16 waves and
one. With C that length the mean is within C v mean|x|. Squares are taken about each wave's own mean and joined about the
row's, so a mean's error e moves the variance by at most 2 e sigma + e^2, and rstd, relatively, by half of that over the
variance; the squares' own sum, of one sign too, rounds by (C + 4) v at most, of which half goes to rstd, and 3 v are its own
quotient, root and addition. y: the errors of both, 4 v of its terms, and u of itself for its type."""
import numpy as np
import pytest
import torch

from oracle import act8
from paper_2608_24070_amd import slim, synth

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
U = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
V = 2.0 ** -24
EPS = 1e-5


def chain(k):
    for most, t, v in ((512, 64, 1), (1024, 64, 2), (4096, 256, 2), (8192, 512, 2), (16384, 512, 4), (32768, 512, 8)):
        if k <= most and (k <= 16384 or k % 8 == 0):
            return 8 * v + 6 + 1 + (t // 64 + 1 if t > 64 else 0)
    return 8 + -(-k // 8192) + 6 + 16 + 1


@pytest.mark.parametrize("k", [100, 512, 1023, 1024, 4096, 5001, 8192, 16383, 16384, 28671, 28672, 32768, 40001])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rms", [False, True])
def test_forward(k, dtype, rms):
    print(f"norm one sign k={k} {dtype} rms={rms}", flush=True)
    rng = synth.stream(40, f"norm/one_sign/{k}")
    x = rng.uniform(1, 2, (6, k)) * 10.0 ** rng.uniform(-3, 3, (6, 1))
    x[3:] = -x[3:]
    t = torch.from_numpy(x.astype(np.float32)).to(DT[dtype])
    g, b = (torch.from_numpy(rng.uniform(0.5, 1.5, k).astype(np.float32)) for _ in range(2))
    y, mean, rstd = slim.norm(t.cuda(), g.cuda(), None if rms else b.cuda(), eps=EPS, rms=rms)
    x, g, b = t.double().numpy(), g.double().numpy(), b.double().numpy()
    ref, mu, rs = act8.norm(x, g, None if rms else b, EPS, rms)
    c, ax = chain(k), np.abs(x).mean(1)
    far = 0.0 if rms else c * V * ax
    if not rms:
        assert np.all(np.abs(mean.double().cpu().numpy() - mu) <= far)
    rel = (c + 4) / 2 * V + 3 * V + far * rs + (far * rs) ** 2
    assert np.all(np.abs(rstd.double().cpu().numpy() - rs) <= rel * rs)
    far, rel, rs = (np.broadcast_to(a, (6,))[:, None] for a in (far, rel, rs))
    d = np.abs(x if rms else x - np.asarray(mu)[:, None])
    terms = d * rs * g + (0 if rms else b)
    lim = U[dtype] * np.abs(ref) + (far * rs * g + rel * d * rs * g + 4 * V * terms) * 1.01
    assert np.all(np.abs(y.double().cpu().numpy() - ref) <= lim)
