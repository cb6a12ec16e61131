"""The layer operators on a GPU at the ends of their ranges.  References in float64; the bounds are test_layer_gpu.py's, with the same
derivation."""
import math

import pytest
import torch

from paper_2607_25234_gb300 import whtmix
from test_layer_gpu import BF, U16, close, phi, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def device():
    whtmix.library()
    torch.cuda.set_device(0)
    yield
    whtmix.sync()


# ---- slopes ----

@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("T,K", [(3, 64), (3, 320), (9729, 64), (9729, 200)])
def test_slopes_of_far_preactivations(T, K, act):
    """act'(p) over all that bf16 holds, each value beside ordinary and beside far ones (two channels share a reciprocal): the
    float32 slope within 2^-16.  One token's dy is 1, all others' 0, so that db is the slope and dw its bf16."""
    far = [5.0, 7.5, 10.0, 16.0, 20.0, 41.0, 64.0, 88.0, 100.0, 200.0, 300.0, 1e3, 1e4, 1e5, 1e6, 1e7, 1e9, 1e19, 1e20, 1e30, 3e38, math.inf]
    far = far + [-v for v in far]
    pairs = [(v, a) for v in far for a in [0.3, -1.0, 2.0, -7.0, 1e3, -1e6, math.inf, -math.inf, math.nan] + rand(7, 8).tolist()]
    p = torch.tensor(pairs + [(a, v) for v, a in pairs], device="cuda").to(BF).view(-1)
    N = p.numel()
    ref = phi(p.double(), act)[1]
    ref[p == math.inf], ref[p == -math.inf] = 1.0, 0.0
    if act != "relu":
        ref[torch.isnan(p)] = math.nan
    dy, x = torch.zeros(T, N, device="cuda").to(BF), torch.zeros(T, K, device="cuda").to(BF)
    dy[1], x[1] = 1.0, 1.0
    w = torch.zeros(N, K, device="cuda").to(BF)
    rows = p.expand(T, N).contiguous()
    if act == "relu":
        rows[torch.isnan(rows)] = 0.5
        ref[torch.isnan(p)] = 1.0
    _, dw, db = whtmix.linear_backward(x, w, dy, rows, act)
    close(db, ref, 2.0 ** -16)
    close(dw, ref[:, None].expand(N, K), 2.0 ** -16 + U16 * (1 + U16) * (ref.abs() + 2.0 ** -16)[:, None])
