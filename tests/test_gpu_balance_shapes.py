"""The balance loss through every way that a token's logits can lie over lanes: four or one logit a lane, one, two, four or sixteen steps, whole and not, up to two experts and up to eight."""
import pytest

from test_gpu_balance import check, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T,E,k", [(70, 4, 2), (70, 5, 2), (70, 12, 1), (70, 9, 8), (70, 64, 4), (70, 68, 2), (70, 128, 2), (70, 128, 5), (70, 100, 2), (70, 252, 3), (70, 516, 2), (70, 65, 6),
                                   (70, 1024, 1), (70, 1021, 2), (2500, 128, 2), (2500, 63, 2), (2500, 100, 3)])
def test_against_64_bits(T, E, k, renorm, dtype):
    print(f"balance T={T} E={E} k={k} renorm={renorm} {dtype}", flush=True)
    z, idx, ds = inputs(T, E, k, T + E + k)
    check(z, idx, 0.01, renorm, 0.5, ds, dtype)
