"""im2win_rms_norm into 8 bits, of fp32 rows: which number is nearest, against arithmetic on whole numbers (64-bit floats cannot tell ties)."""
import pytest
import torch

from paper_2608_20725_b200 import binding

pytestmark = pytest.mark.gpu


def nearest(h, w):
    """127 h w / top to the nearest number, ties to the even one, of lists of whole numbers."""
    z = [a * b for a, b in zip(h, w)]
    top = max(abs(x) for x in z)
    out = []
    for x in z:
        n, rest = divmod(254 * abs(x) + top, 2 * top)          # floor(127 |x| / top + 1/2)
        n -= rest == 0 and n % 2 == 1
        out.append(n if x >= 0 else -n)
    return out


def test_the_oracle_of_whole_numbers():
    assert nearest([11020298, 9935623], [9427443] * 2) == [127, 114]
    assert nearest([13409422, 12828699], [8717249] * 2) == [127, 122]
    assert nearest([254, 1, 3, -3, -1, 0], [1] * 6) == [127, 0, 2, -2, 0, 0]


@pytest.mark.parametrize("weight", [1, 9427443, 8717249, 16777215, 10000019])
@pytest.mark.parametrize("channels", [512, 509, 8192])
@pytest.mark.parametrize("exponent", [0, -70])
def test_fp32_halves_are_seen_exactly(weight, channels, exponent):
    """top = 254 t, others (2 r + 1) t: quotients of whole numbers and a half, and those of the next numbers on either side.  With an exponent of
    -70 for both the products lie below what fp32 holds exactly."""
    gen = torch.Generator().manual_seed(channels + weight)
    rows = []
    for _ in range(6):
        t = int(torch.randint(20000, 66000, (1,), generator=gen)) | 1
        r = torch.randint(0, 127, (channels,), generator=gen)
        row = ((2 * r + 1) * t + torch.randint(-1, 2, (channels,), generator=gen)) * (1 - 2 * torch.randint(0, 2, (channels,), generator=gen))
        row[0] = 254 * t
        rows.append([int(x) for x in row.clamp(-254 * t, 254 * t)])
    want = torch.tensor([nearest(row, [weight] * channels) for row in rows], dtype=torch.int8)
    x = torch.tensor(rows, dtype=torch.float64).mul(2.0 ** exponent).float().cuda()
    w = torch.full((channels,), float(weight)).mul(2.0 ** exponent).cuda()
    y, scales = torch.zeros(6, channels, dtype=torch.int8, device="cuda"), torch.zeros(6, device="cuda")
    binding.im2win_rms_norm(x, w, y, scales=scales)
    assert torch.equal(y.cpu(), want)
