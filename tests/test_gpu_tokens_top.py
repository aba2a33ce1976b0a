"""The best alternatives where the waves of a block select by themselves: orders that
raise a wave's bound in every tile or never, ties within and across waves and tiles,
one wave that holds all of the best, masks, NaN, every share of a wave."""
import numpy as np
import pytest

from test_gpu_tokens import native_mod, torch_type

pytestmark = pytest.mark.gpu

ORDERS = ["rising", "falling", "equal", "three", "one wave", "one tile", "masked", "nan", "normal"]


def rows(rng, how, n, v, elems):
    """n rows of v values that every type holds; elems: of a 16-byte vector."""
    x = rng.integers(-512, 512, (n, v)).astype(np.float32) / 64
    at = np.arange(v)
    wave = at // (64 * elems) % 4  # of a block's four, in every tile of 1024 vectors
    tile = at // (1024 * elems)
    if how == "rising":
        x = np.broadcast_to(np.floor(at * (256.0 / v)), (n, v)) + rng.integers(0, 2, (n, 1))
    elif how == "falling":
        x = np.broadcast_to(-np.floor(at * (256.0 / v)), (n, v)) - rng.integers(0, 2, (n, 1))
    elif how == "equal":
        x[:] = 0.5
    elif how == "three":
        x = rng.integers(0, 3, (n, v)).astype(np.float32)
    elif how == "one wave":
        x += 32.0 * (wave == rng.integers(0, 4, (n, 1)))
    elif how == "one tile":
        x += 32.0 * (tile == rng.integers(0, tile[-1] + 1, (n, 1)))
    elif how == "masked":
        x[rng.random((n, v)) < 0.999] = -np.inf
        x[1] = -np.inf
    elif how == "nan":
        x[rng.random((n, v)) < 0.01] = np.nan
        x[1, 5:] = np.nan
    return np.ascontiguousarray(x)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("how", ORDERS)
@pytest.mark.parametrize("n,tiles,more", [(520, 3, 5), (1027, 2, 1), (2050, 2, 3), (520, 0, 777)])
def test_alternatives(gpu, dtype, how, n, tiles, more):
    import torch

    native = native_mod()
    elems = 4 if dtype == "f32" else 8
    v = tiles * 1024 * elems + more
    rng = np.random.default_rng(n + v)
    z = torch.from_numpy(rows(rng, how, n, v, elems)).to(gpu, torch_type(dtype))
    # largest first, ties to the lowest index, NaN behind everything
    key = torch.where(z.isnan(), torch.full_like(z.float(), -float("inf")), z.float())
    order = torch.sort(torch.where(z.isnan(), key, key.clamp_min(-1e30)), dim=1, descending=True,
                       stable=True).indices
    for top in (1, 2, 3, 5, 7, 20, 64, 65, 128):
        f = native.pdb_token_logprobs(z, top=top)
        assert torch.equal(f.top_id.long(), order[:, :top]), (top, how)
        got = f.top_logp
        if how == "nan":
            assert bool(got[z.isnan().any(dim=1)].isnan().all())
        else:
            want = z.gather(1, order[:, :top]).double() - z.double().logsumexp(1, keepdim=True)
            want = want.masked_fill((z == -float("inf")).all(dim=1, keepdim=True), -float("inf"))
            same = (got.double() == want) | ((got.double() - want).abs() <= 1e-4)
            assert bool(same.all()), (top, how)
