"""The embedding gradient's order of many tokens: digits of every width, tables whose
rows fill their digits or just pass them, tiles of the sort from partly filled to all
full, hot tokens, padding, both index types."""
import numpy as np
import pytest

import tokenref as ref
from test_gpu_tokens import check, f64, native_mod

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,v,d", [
    (6144, 1023, 3), (6145, 1023, 3), (6145, 1024, 3), (12289, 1023, 3), (12289, 1024, 3),
    (65537, (1 << 18) - 1, 2), (131073, 1 << 18, 2), (262144, (1 << 19) + 3, 1),
    (200001, (1 << 20) - 1, 2), (1100003, 1 << 20, 1), (2097152, 700001, 2), (262145, 70001, 3),
    (4194304, 40000, 1), (4194305, 900, 1), (200003, (1 << 25) + 5, 1), (8388608, 1500, 1)])
@pytest.mark.parametrize("how", ["uniform", "hot", "one"])
def test_embed_grad_order(gpu, n, v, d, how):
    import torch

    native = native_mod()
    rng = np.random.default_rng(n + v)
    tok = rng.integers(0, v, n)
    if how == "hot":  # half of the positions share two tokens, the table's ends are in use
        at = rng.random(n)
        tok[at < 0.3] = v - 1
        tok[(at > 0.3) & (at < 0.5)] = v // 3
        tok[at > 0.95] = -1
        tok[n // 2] = 0
    elif how == "one":
        tok[:] = v - 1
    # 32-bit inputs made as such: what the sums are of is known exactly
    dy = rng.normal(size=(n, d)).astype(np.float32)
    old = np.zeros((v, d), np.float32)
    want, bound = ref.embed_grad(dy.astype(np.float64), tok, old, 1.0, False)
    dyg = torch.from_numpy(dy).to(gpu)
    for index in (torch.int32, torch.int64):
        tg = torch.from_numpy(tok).to(gpu, index)
        status = torch.zeros(1, dtype=torch.int32, device=gpu)
        got = native.pdb_embed_grad(dyg, tg, torch.full((v, d), 5.0, device=gpu), status=status)
        check(f64(got), want, bound, "grad")
        assert int(status) == native.PDB_OK
        tg[n // 7] = v  # one token out of range: said so, and left out
        less, _ = ref.embed_grad(dy[n // 7:n // 7 + 1].astype(np.float64), tok[n // 7:n // 7 + 1],
                                 np.zeros((v, d), np.float32), 1.0, False)
        got = native.pdb_embed_grad(dyg, tg, torch.full((v, d), 5.0, device=gpu), status=status)
        check(f64(got), want - less, bound, "grad without it")
        assert int(status) == -1


def test_rows_wider_than_a_grid_of_narrow_groups(gpu):
    """Tokens that cross blocks, in rows of over 2^21 columns."""
    import torch

    native = native_mod()
    n, v, d = 300, 3, (1 << 21) + 3
    tok = torch.arange(n, device=gpu) * v // n
    dy = torch.ones(n, d, device=gpu)
    dy[:, 1::2] = 2.0
    got = native.pdb_embed_grad(dy, tok, torch.full((v, d), 7.0, device=gpu))
    assert torch.equal(got, dy[:v] * (n // v))
