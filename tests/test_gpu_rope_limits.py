"""The rotation at the most tokens of one call.  Oracle and tolerance are those
of test_gpu_rope."""
import pytest

torch = pytest.importorskip("torch")

from paper_2510_14126_amd import binding as pa  # noqa: E402
from test_gpu_rope import DEV, EPS, check, rotation  # noqa: E402

pytestmark = pytest.mark.gpu


def test_most_tokens():
    print("[gpu case] norm_rope most tokens", flush=True)
    n, d = 2 ** 26 - 64, 16
    rope, freqs, magnitude = rotation(d, d, 0)
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(n, d, generator=gen, device=DEV, dtype=torch.bfloat16)
    out = torch.zeros_like(x)
    pos = torch.arange(n, device=DEV, dtype=torch.int32)
    pa.paged_attn_norm_rope(rope, x, d, 1, None, None, 0, 0, None, EPS, pa.PA_BF16, pos, n, out, d, None, 0)
    torch.cuda.synchronize()
    for a in (0, n // 2 - 5, n - 3000):
        rows = slice(a, a + 3000)
        check(out[rows].view(-1, 1, d), x[rows].view(-1, 1, d), None, pos[rows].cpu().numpy(), freqs, magnitude, False,
              torch.bfloat16, 25)      # a position's product with its frequency: 2^26 2^-53 radians, below one step more
    assert not (out == 0).all(-1).any()
