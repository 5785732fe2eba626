"""What the tests of the operators around a served cache share: derived bounds and small caches."""
import numpy as np
import torch

from oracle import decode_oracle as D

DEV = "cuda:0"
U24 = 2.0 ** -24                # half a step of fp32


def f64(t):
    return t.detach().double().cpu().numpy()


def weight_error(d, big, lse, keys):
    """Bound of the relative error of a softmax weight or of a sum of `keys` of them in fp32: d roundings of a logit, none larger
    than half a step of the sum of its products' magnitudes `big`; the multiplication by scale * log2(e), a constant with its
    own rounding, and the subtraction of the reference, at the size of a logit (at most |lse| + ln(keys) + 2 big) each;
    two units in the last place of the exponential; and a sum in any order."""
    size = np.abs(lse) + np.log(np.maximum(keys, 1)) + 2 * big
    return d * U24 * big + 4 * U24 * size + 4 * U24 + keys * U24


def attention_bound(dtype, d, ref, mag, big, lse, keys, rounded):
    """|error| of an output element: its weights' errors (twice: numerator and sum), the products' and their sum's rounding, the
    division; for `rounded` outputs half a step of the type for the weights of the second product and half a
    step for the result (and, in fp16, half of the smallest step of a weight: 2^-32 of the largest)."""
    rel = 2 * weight_error(d, big, lse, keys)[..., None] + (np.asarray(keys)[..., None] + 4) * U24
    bound = rel * mag + 2 * U24 * np.abs(ref) + 1e-37
    if rounded and dtype != torch.float32:
        half = torch.finfo(dtype).eps / 2
        bound = bound + half * mag * 1.01 + half * (np.abs(ref) + bound)
        if dtype == torch.float16:
            bound = bound + np.asarray(keys)[..., None] * 2.0 ** -31 * mag.max() + 2.0 ** -25
    return bound


def lse_bound(d, big, lse, keys):
    return weight_error(d, big, lse, keys) + 4 * U24 * np.abs(lse) + 4 * U24


def assert_within(got, ref, bound, what):
    got, ref = np.asarray(got, dtype=np.float64), np.asarray(ref)
    assert got.shape == ref.shape, what
    assert np.isfinite(got).all(), f"{what}: not finite"
    over = np.abs(got - ref) / bound
    print(f"  {what}: error at most {over.max():.3f} of its bound", flush=True)
    assert over.max() <= 1.0, f"{what}: {int((over > 1).sum())} of {over.size} beyond their bound, worst {over.max():.2f} times"


def offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)])


def segments(t, cu, headroom, lens):
    """The held rows of each segment."""
    start = D.segment_starts(cu, headroom)
    return [t[start[s]:start[s] + int(lens[s])] for s in range(len(lens))]
