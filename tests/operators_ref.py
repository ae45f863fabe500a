"""What the tests of the operators beside the Update stage share: inputs, strided rows, and how far a rounded result may lie from the
value in 64 bits.  Holds no arithmetic of the library's."""
import torch

DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS32 = 2.0 ** -24                       # half a unit in the last place of fp32, relative
# of a value, relative: bf16 keeps 8 significant bits, fp16 11, fp32 24
HALF_ULP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
FLOOR = {"bf16": 2.0 ** -133, "f16": 2.0 ** -25, "f32": 2.0 ** -149}        # half the smallest subnormal


def code(paro, dtype):
    return {"bf16": paro.PARO_BF16, "f16": paro.PARO_F16, "f32": paro.PARO_F32}[dtype]


def rng(seed):
    return torch.Generator().manual_seed(seed)


def rows(n, width, pad, dtype, fill=float("nan")):
    """A device buffer of n rows, `pad` elements apart, that starts at an odd element when pad is odd; and the view of its rows."""
    whole = torch.full((n * (width + pad) + 64,), fill, dtype=TORCH[dtype], device=DEV)
    at = 1 if pad % 2 else 0
    return whole, whole[at:at + n * (width + pad)].view(n, width + pad)[:, :width]


def put(values, pad, dtype):
    """Rows on the device with these values (rounded to the dtype), NaN in between; and what they hold, in 64 bits on the host."""
    _whole, view = rows(values.shape[0], values.shape[1], pad, dtype)
    view.copy_(values.to(TORCH[dtype]))
    return view, values.to(TORCH[dtype]).double()


def rounding(ref, dtype, err):
    """Bound on |result - ref|: an error of the fp32 value before it is rounded, the rounding of that, and its subnormals."""
    return err + HALF_ULP[dtype] * (ref.abs() + err) + FLOOR[dtype]


def check(got, ref, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == ref.shape, what
    same = (got == ref) | (got.isnan() & ref.isnan())          # infinities and NaN have to be where the reference has them
    finite = ref.isfinite()
    bad = ~same & (~finite | ~((got - torch.where(finite, ref, 0.0)).abs() <= bound))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: " \
        f"{got[bad][0].item()} for {ref[bad][0].item()}"


def stream():
    return torch.cuda.current_stream().cuda_stream


def workspace(size):
    """Filled with garbage: its contents must be of no account."""
    return torch.full((size,), 0xA5, dtype=torch.uint8, device=DEV)
