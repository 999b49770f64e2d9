"""Log probabilities where logits over the temperature are large: small temperatures, rows masked with finite
numbers, values and temperatures near fp32's limits, against 64 bits.

The bounds are test_gpu_logprobs's, and hold over this range.  Between maxima, for the asked token, and in the
sums of a maximum m far from 0, an exponent is (x - m) k, or that with x and m halved: a rounding of the
difference and one of the product, u |d| each.  In other sums (|m k| < 2^20) it is x k - M with one
rounding, M being m k rounded, and the sum is then taken times 2^(M - m k), an exponential like the others (and
the sum of exponents freed of M - m k, 2^-5 at most: a rounding of the size of H + 1 more).  With the three roundings
of k an exponent is within 5 u |d| of itself, whatever the size of m k."""
import pytest
import torch

from test_gpu_logprobs import call, check_items

pytestmark = pytest.mark.gpu


def large_rows(V, dev):
    """Rows all at a large number, around it, masked with it, and with 16 bytes of it."""
    g = torch.Generator(device=dev)
    g.manual_seed(V)
    n = lambda: torch.randn(V, device=dev, generator=g)  # noqa: E731
    a = torch.arange(V, dtype=torch.float32, device=dev)
    rows = {}
    for c in (1e6, -1e6, -1e9, -1e10, -1e12, 1e20, -1e20, -1e32):
        rows["all", c] = torch.full((V,), c, device=dev)
        rows["around", c] = c * (1 + 2.0 ** -20 * n())
        rows["masked", c] = torch.where(torch.rand(V, device=dev, generator=g) < 0.9, c, 3 * n())
        rows["one allowed", c] = torch.where(a == V // 2, 1.5, c)
        rows["first", c] = torch.where(a < 8, c, 3 * n())
        rows["one group", c] = torch.where((a >= 16) & (a < 24), c, 3 * n())
    for s in (1, -1):   # |m k| on both sides of 2^20 at temperature 1
        rows["up", s] = s * 726817 + (a - V // 2) / 16
        rows["down", s] = s * 726817 - (a - V // 2) / 16
        rows["beside", s] = s * 726817 + (a - V // 2) / V
    rows["0 and far"] = torch.where(a % 5 == 0, -726817.0, 0.0)
    return torch.stack(list(rows.values()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [5, 40, 3001, 40000])
def test_small_temperatures(cuda_device, V, dtype):
    from paper_2405_18628_gb300 import ppd
    g = torch.Generator(device=cuda_device)
    g.manual_seed(V)
    for temperature in (1e-2, 1e-3, 1e-4, 1e-5, 1e-6, 1e-7, 1e-8, 1e-9, 1e-10, 1e-20, 1e-38):
        logits = (20 + 3 * torch.randn(1, 3, V, device=cuda_device, generator=g)).to(dtype)
        logits[0, 2] = 12.625 - logits[0, 2].float().abs()
        tokens = logits.argmax(-1).int()
        tokens[0, 1] = V - 1
        check_items(call(ppd, logits, tokens, temperature, K=3), logits, tokens, temperature, None, [(0, 0), (0, 1), (0, 2)])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("temperature", [1.0, 0.8, 0.5, 0.1])
@pytest.mark.parametrize("V", [5, 40, 3001, 40000])
def test_large_values_and_finite_masks(cuda_device, V, temperature, dtype):
    from paper_2405_18628_gb300 import ppd
    logits = large_rows(V, cuda_device)[None].to(dtype)
    T = logits.shape[1]
    for pick in (0, V // 2, V - 1):
        tokens = torch.full((1, T), pick, dtype=torch.int32, device=cuda_device)
        check_items(call(ppd, logits, tokens, temperature, K=3), logits, tokens, temperature, None, [(0, i) for i in range(T)])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("temperature", [1e5, 1e25, 1e30, 1e34, 1e37, 3e38])
def test_large_temperatures(cuda_device, temperature, dtype):
    """Differences past fp32's range whose exponents are not."""
    from paper_2405_18628_gb300 import ppd
    V = 3001
    a = torch.arange(V, dtype=torch.float32, device=cuda_device)
    g = torch.Generator(device=cuda_device)
    g.manual_seed(7)
    rows = [torch.where(a % 7 == 3, 3.0e38, -3.0e38), torch.where(a % 7 == 3, -3.0e38, 2.0e38), torch.full((V,), -3.4028234e38, device=cuda_device),
            1e38 * torch.randn(V, device=cuda_device, generator=g).clamp(-3.3, 3.3), torch.where(a < 9, a, -3.3e38), a, 1e6 * a]
    logits = torch.stack(rows)[None].to(dtype)
    logits = torch.where(logits == float("-inf"), -3.3e38, logits)   # (rounded past the type's range)
    T = len(rows)
    for pick in (0, 3, V - 1):
        tokens = torch.full((1, T), pick, dtype=torch.int32, device=cuda_device)
        check_items(call(ppd, logits, tokens, temperature, K=5), logits, tokens, temperature, None, [(0, i) for i in range(T)])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V,K", [(2600, 5001, 0), (2600, 5001, 20), (2600, 5001, 32), (2000, 5001, 5), (2000, 5001, 21), (5200, 5001, 20), (5200, 301, 32), (1000, 2048, 20),
                                   (1000, 4097, 20)])
def test_blocks_of_every_size(cuda_device, n, V, K, dtype):
    """The same rows, first and last, where blocks of every size take them."""
    from paper_2405_18628_gb300 import ppd
    g = torch.Generator(device=cuda_device)
    g.manual_seed(V + K)
    large = large_rows(V, cuda_device)
    h = len(large)
    logits = (20 + 3 * torch.randn(n, V, device=cuda_device, generator=g)).to(dtype)
    logits[:h] = logits[n - h:] = large.to(dtype)
    logits, tokens = logits[None], torch.randint(0, V, (1, n), device=cuda_device, generator=g).int()
    tokens[0, n - h:] = tokens[0, :h]
    for temperature in (0.8, 1e-8):
        r = call(ppd, logits, tokens, temperature, K=K)
        check_items(r, logits, tokens, temperature, None, [(0, i) for i in [*range(h), h, n // 2, *range(n - h, n)]])
