"""The operators in front of attention and over shared caches together, as a server uses them: a document's prompt is normed, turned,
attended, compressed and kept once; several continuations share it, each token normed and turned in front of its step."""
import numpy as np
import pytest
import torch

import paper_2407_11550_amd as adakv
from oracle import serve_oracle as S
from serve_util import DEV, attention_bound, f64, lse_bound

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,many", [(torch.bfloat16, 3), (torch.bfloat16, 20), (torch.float16, 9), (torch.float32, 5)])
def test_continuations_of_a_compressed_prompt(dtype, many):
    """Against forks of the cache (cache_move) with the plain step, and against 64 bits."""
    n, w, h_q, h, d, headroom, tokens = 900, 16, 8, 2, 64, 6, 4
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=DEV).to(dtype)

    layer = adakv.Layer(dtype, h_q, h, d, w, 7, 0.2, [n], [h * 250])
    rot = adakv.Rotary(d, base=500000.0, scaling="parts", factor=4.0, original_len=512, magnitude=1.1)
    qw, kw = randn(d).abs() + 0.5, randn(d).abs() + 0.5
    fused = randn(n + w, (h_q + 2 * h) * d)
    q, k, v = (fused[:, a * d:b * d].view(n + w, b - a, d) for a, b in ((0, h_q), (h_q, h_q + h), (h_q + h, h_q + 2 * h)))
    q, k = adakv.norm_rotary(layer, rot, q, k, qw, kw)
    _, lse = adakv.window_attn(layer, q, k, v.contiguous(), n + w, want_lse=True)
    made = adakv.compress(layer, q[n:].transpose(0, 1).contiguous().view(1, h_q, w, d), k, v.contiguous(), row_lse=lse)
    cu = made["cu_seqlens"]
    Kp, Vp, p_len = adakv.cache_build(layer, k, v.contiguous(), made["indices"], cu, 0)
    # kept once, and an own cache of one spare row and head-room for each continuation
    own = adakv.Layer(dtype, h_q, h, d, 1, 7, 0.2, [n] * many, [h] * many)
    cu_own = torch.arange(many * h + 1, dtype=torch.int32, device=DEV)
    rows = adakv.cache_rows(own, headroom)
    K, V, lens = torch.zeros(rows, d, dtype=dtype, device=DEV), torch.zeros(rows, d, dtype=dtype, device=DEV), torch.zeros(many * h, dtype=torch.int32, device=DEV)
    prefix = adakv.Prefix(layer, cu, 0, Kp, Vp, p_len, [0] * many)
    # the same as forks
    forks, cu_f, Kf, Vf, len_f = adakv.cache_move(layer, [0] * many, cu, 0, Kp, Vp, p_len, headroom)
    for t in range(tokens):
        q_new, k_new, v_new = randn(many, h_q, d), randn(many, h, d), randn(many, h, d)
        pos = torch.full((many,), n + w + t, dtype=torch.int32, device=DEV)
        q_new, k_new = adakv.norm_rotary(own, rot, q_new, k_new, qw, kw, positions=pos)
        out, lse = adakv.decode_prefix_step(own, q_new, k_new, v_new, cu_own, headroom, K, V, lens, prefix, want_lse=True)
        out_f, lse_f = adakv.decode_step(forks, q_new, k_new, v_new, cu_f, headroom, Kf, Vf, len_f, want_lse=True)
        assert (lens == t + 1).all()
        c0 = cu.cpu().numpy()
        for b in (0, many - 1):
            for c in range(h):
                s = b * h + c
                a = s * (1 + headroom)
                Ks = f64(torch.cat([Kp[c0[c]:c0[c + 1]], K[a:a + t + 1]]))
                Vs = f64(torch.cat([Vp[c0[c]:c0[c + 1]], V[a:a + t + 1]]))
                for i in range(c * 4, c * 4 + 4):
                    ref, z, mag, big = S.attend(f64(q_new[b, i]), Ks, Vs, d ** -0.5)
                    keys = np.array(len(Ks))
                    bound = attention_bound(dtype, d, ref, mag, np.array(big), np.array(z), keys, rounded=False) + mag * 2.0 ** -23
                    if dtype == torch.float16:
                        bound = bound + len(Ks) * 2.0 ** -45 * np.abs(Vs).max()
                    z_bound = lse_bound(d, np.array(big), np.array(z), keys)
                    for o, l, what in ((out, lse, "shared"), (out_f, lse_f, "forked")):
                        assert (np.abs(f64(o[b, i]) - ref) <= bound).all(), (what, t, b, i)
                        assert abs(float(l[b, i]) - z) <= z_bound, (what, t, b, i)
