"""The norm without an eps: rows of zeros, and rows whose squares leave the range of 32 bits below."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_clear import TYPES, U32, ctx, gen, half_step, norm_reference, strided  # noqa: E402, F401


@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-36, 1e-12])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows, d", [(7, 40), (7, 1000), (7, 2560), (2100, 2560), (1100, 3001), (7, 8191), (7, 20001)])
def test_small_rows(ctx, rows, d, kind, eps):
    """Rows of 2^-8 to 2^-140 and of zeros in turn; the sum goes to x's place, to the residual's, or nowhere, and the results are those of the rows as they are."""
    g = gen(rows + d)
    x, gain = torch.randn(rows, d, generator=g), (1 + 0.2 * torch.randn(d, generator=g)).to(TYPES[kind])
    for i, e in enumerate((-8, -49, -52, -70, -100, -140)):
        x[i::7] *= 2.0 ** e
    x[6::7] = 0
    x = x.to(TYPES[kind])
    r = x.roll(1, 1) * 0.5
    for residual, into in ((None, None), (r, None), (r, "x"), (r, "residual")):
        h = norm_reference(x, gain, residual, eps)[0]
        up = np.where(np.abs((h.float() * gain.float()).numpy()).max(1, keepdims=True) < 2.0 ** -100, np.float32(2.0 ** 100), np.float32(1))  # 1 / most would be infinite
        p = (h.float() * gain.float()).numpy() * up
        most = np.abs(p).max(1, keepdims=True)
        codes = np.where(most > 0, np.rint(p * (np.float32(127) * (np.float32(1) / np.where(most > 0, most, np.float32(1))))), 0)
        # products are held in 32 bits, which round them below the normal range; then the norm in 64, rows of zeros 0
        p64, dark = torch.from_numpy(p).double() / torch.from_numpy(up).double(), (h == 0).all(1, keepdim=True)
        full = torch.where(dark, 0.0, p64 / torch.sqrt((h.double() ** 2).mean(1, keepdim=True) + eps))
        scales = full.abs().amax(1) / 127
        xd, rd = strided(x, 3), None if residual is None else strided(r, 3)
        out = strided(torch.zeros_like(x), 1)
        got, got_scales = ctx.clear_norm(xd, gain.cuda(), residual=rd, eps=eps, sum_out={"x": xd, "residual": rd, None: None}[into], out=out, codes=torch.empty(rows, d, dtype=torch.int8, device="cuda"))
        assert np.array_equal(got.cpu().numpy(), codes)
        near = 64 * U32  # as in test_norm; eps in 32 bits half a step more (a whole one where it is the smallest number)
        near = near + (abs(float(np.float32(eps)) - eps) / eps if eps else 0)
        smallest = 2.0 ** -149
        assert ((got_scales.cpu().double() - scales).abs() <= near * scales + 2 * smallest).all()
        least = torch.finfo(TYPES[kind]).smallest_normal * half_step(kind) * 2
        assert ((out.cpu().double() - full).abs() <= (near + half_step(kind)) * full.abs() + least).all()
        if into:
            assert torch.equal({"x": xd, "residual": rd}[into].cpu(), h)
