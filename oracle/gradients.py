"""The norm of many gradients and the clipping by it, in 64 bits."""
import numpy as np


def norm(tensors):
    """tensors: arrays [parts, n].  (norm of all, [norm of each])."""
    squares = [float(np.sum(np.asarray(t, dtype=np.float64).sum(axis=0) ** 2)) for t in tensors]
    return float(np.sqrt(np.sum(squares))), np.sqrt(squares)


def scale(total, max_norm):
    if not np.isfinite(total):
        return float("nan")
    return max_norm / total if total > max_norm else 1.0
