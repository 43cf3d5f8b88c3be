"""The clear product as the reference of the encrypted one: the codes of a norm, encrypted, multiplied with the same ternary weights and decrypted."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import workloads as wl  # noqa: E402
from helpers import Pair  # noqa: E402


def test_a_decrypted_product_is_the_clear_one():
    w = wl.WORKLOADS[0]
    p = Pair(w.param_tuple())
    rng = wl.rng_for(w.index)
    W = wl.ternary_weights(rng, w.d_in, w.d_out)
    x = torch.from_numpy(rng.standard_normal((w.tokens, w.d_in))).float().cuda()
    codes, scales = p.ctx.clear_norm(x, torch.full((w.d_in,), 0.25, device="cuda"))
    weights = p.ctx.clear_weights_prepare(W, np.ones(w.d_out, dtype=np.float32))
    clear = p.ctx.clear_matmul(weights, codes, scales, dtype=torch.float32).cpu().double().numpy()
    X = codes.cpu().double().numpy() * scales.cpu().double().numpy()[:, None]
    _, ct = p.encrypt_both(wl.pack_columns(X, p.n), p.pr.L)
    _, gk = p.galois_keys([r * w.tokens for r in range(1, w.c_tot)])
    out = p.ctx.ternary_matmul(gk, ct, w.tokens, w.d_in, W, w.placement)
    dec = p.ctx.decrypt(p.g_sk, out)
    got = np.stack([dec[i, (i % w.c_tot) * w.tokens:(i % w.c_tot + 1) * w.tokens] for i in range(w.d_out)], 1)
    # the encryption's noise on this ring stays below 1e-3; the clear product is a whole number times a scale, rounded twice
    assert np.abs(got - clear).max() < 1e-3 + 2 * 2.0 ** -24 * np.abs(clear).max()
    assert np.abs(clear).max() > 1
    weights.free()
    p.close()
