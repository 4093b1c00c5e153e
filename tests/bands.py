"""Whether an output lies within a tolerance of the exact value."""
import torch


def outside(got, want, tol):
    """Where `got` is neither within tol of want (fp64) nor, in bf16, the
    rounding of a value that is."""
    if got.dtype == torch.bfloat16:
        low, high = (want - tol).float().bfloat16(), (want + tol).float().bfloat16()
        return ~((got >= low) & (got <= high))
    return ~((got.double() - want).abs() <= tol)
