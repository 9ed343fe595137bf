"""Shared helpers of the attention block's tests: device copies, and the check of a result against float64."""
import numpy as np
import torch

U32 = 2.0 ** -24                          # half a step of float32, relative
UBF = torch.finfo(torch.bfloat16).eps / 2  # of bfloat16


def rounded(a, dtype):
    """The values that a tensor of this type can hold, in float64."""
    return torch.as_tensor(np.ascontiguousarray(a)).to(torch.bfloat16 if dtype == "bf16" else torch.float32).double().numpy()


def dev(a, dtype="f32"):
    if a is None:
        return None
    t = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "u8": torch.uint8}[dtype]
    return torch.as_tensor(np.ascontiguousarray(a)).to(t).cuda()


def empty(shape, dtype="f32", fill=float("nan")):
    """A device tensor filled with what no result is."""
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    return torch.full(shape if isinstance(shape, tuple) else (shape,), fill, dtype=t, device="cuda")


def room(n):
    """A workspace of exactly n bytes, with a guard behind it that must stay as it is."""
    t = torch.full((int(n) + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    return t[:int(n)], t[int(n):]


def untouched(*guards):
    return all(bool((g == 0xA5).all()) for g in guards)


def close(name, got, want, mag, steps, dtype="f32"):
    """|got - want| <= steps half-steps of float32 of the magnitude that the result is made of, and half a step of its own type."""
    got = got.double().cpu().numpy().reshape(want.shape) if isinstance(got, torch.Tensor) else got
    assert np.isfinite(got).all(), name
    tol = steps * U32 * mag + (UBF * (np.abs(want) + steps * U32 * mag) if dtype == "bf16" else 0.0) + 1e-37
    bad = np.abs(got - want) > tol
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, worst {np.max(np.abs(got - want) / tol):.3g} of what is allowed"
