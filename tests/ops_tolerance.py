"""How far the weights of a routing may be off, weight by weight."""
import numpy as np

U = 2.0 ** -24


def route_weights(z, ids, want, sigmoid):
    """z [T, E] logits, ids, want [T, k] -> [T, k].  The exponential's argument (a difference to the row's largest logit, or the logit)
    is rounded once, and its error grows with the argument: of the chosen ones that have a score at all, the largest counts, since they share
    a sum.  Exponential, sums over the experts and over the chosen, quotients and scale: 40 roundings.  What is left is below the normal
    numbers of 32 bits."""
    z = np.where(np.isnan(z), -np.inf, np.asarray(z, np.float64))
    top = np.zeros((len(z), 1)) if sigmoid else z.max(axis=1, keepdims=True)
    with np.errstate(invalid="ignore"):
        arg = np.abs(np.take_along_axis(z - top, ids, 1))
    arg = np.where(np.isfinite(arg) & (want > 0), arg, 0).max(axis=1, keepdims=True)
    return want * (arg + 40) * U + 1e-37
