"""The sums of the draft head over 4-bit weights, on products of one sign, where every addition that is cut off or rounded shows.

Tolerances, from the order in which the kernels add.
bfloat16: the products of 16 elements are added to a sum by one tensor-core instruction, which aligns 17 numbers to the largest and may
cut each off below float32's last place: 17 * 2^-23 of the sum so far at most.  A sum begins again after C instructions: 64 (8 blocks of 128 elements),
or as many as there are, with every other block where two warps issue (up to 64 rows).  With products of like size the sum so far is half of its end on
average, so a chain is off by 17 * 2^-23 * (C + 1) / 2 of itself, and so are all chains of their total.  The chains' ends are then added in rounded
float32, two additions for each of the S stretches (2^-24 each, of the total at most).
That is a bound for the worst alignment.  That sums do begin again shows in comparison: chains of long and of short rows are then as long, and off as
far, but for the additions of the S stretches (without, a row of 131072 elements would be off 64 times as far as one of 2048).
float32: a lane adds the products of a quarter of the elements in turn (2^-24 each, half of that on average over growing sums), then the four
quarters and, of panels that warps share, sixteen parts.
The log-sum-exp moves by the largest such error; its exponentials and sums stay below 3e-5."""
import numpy as np
import pytest
import torch

import q4_util as u
import test_gpu_q4_draft as draft

pytestmark = pytest.mark.gpu


def bound(dtype, M, H):
    if dtype == "fp32":
        return (H / 8 + 1 + 2 + 16) * 2.0 ** -24
    blocks = (H + 127) // 128
    issuers = 2 if M <= 64 else 1
    C = min(8, (blocks + issuers - 1) // issuers) * 8
    S = (blocks + 8 * issuers - 1) // (8 * issuers)
    return 17 * 2.0 ** -23 * (C + 1) / 2 + 2 * S * 2.0 ** -24


def run(dtype, M, H, V):
    """Largest relative error of a logit, and the case."""
    rng = np.random.default_rng([M, H])
    c = draft._Case(dtype, M, H, V, 2, 2, 64, weights=rng.uniform(0.25, 0.75, size=(2, V + 1, H)) * 8 / H, bias=False)
    c.x = torch.from_numpy(rng.uniform(0.5, 1.5, size=(M, H)).astype(np.float32)).to(u.DEV, u.act_of(dtype))
    c.run()
    assert c.h.poll_status() == 0
    z, _ = c.reference()
    assert float(z.min()) > 1.0
    return ((c.z.double() - z).abs() / z).max().item(), c, z


@pytest.mark.parametrize("dtype,M,H,V", [("bf16", 1, 128, 200), ("bf16", 1, 1032, 200), ("bf16", 2, 2048, 300), ("bf16", 16, 8192, 300), ("bf16", 33, 32768, 60),
                                         ("bf16", 1, 131072, 40), ("bf16", 70, 2056, 100), ("bf16", 100, 16384, 60), ("fp32", 1, 256, 300),
                                         ("fp32", 4, 4096, 100), ("fp32", 1, 40000, 20)])
def test_sums_of_products_of_one_sign(dtype, M, H, V):
    off, c, z = run(dtype, M, H, V)
    assert off <= bound(dtype, M, H)
    assert torch.all((c.out[2].double() - torch.logsumexp(z, -1)).abs() <= bound(dtype, M, H) * z.amax(-1) + 3e-5)


@pytest.mark.parametrize("M", [1, 70])
def test_long_rows_are_off_as_far_as_short_ones(M):
    short, long = run("bf16", M, 2048, 300)[0], run("bf16", M, 131072, 40)[0]
    stretches = 131072 // (128 * 8 * (2 if M <= 64 else 1))
    assert long <= 3 * short + 2 * stretches * 2.0 ** -24          # (3: the largest of other draws)
