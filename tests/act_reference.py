"""The activations and their slopes in 64 bits, and how far the kernels' may be from them."""
import numpy as np
from scipy.special import erfc, expit

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
_A, _B = np.sqrt(8 / np.pi), 0.044715


def value(z, act):
    z = np.asarray(z, dtype=np.float64)
    if act == "relu":
        return np.maximum(z, 0)
    if act == "gelu":
        return 0.5 * z * erfc(-z / np.sqrt(2))
    if act == "gelu_tanh":
        return z * expit(_A * (z + _B * z ** 3))
    if act == "silu":
        return z * expit(z)
    return z


def slope(z, act):
    z = np.asarray(z, dtype=np.float64)
    if act == "relu":
        return (z > 0).astype(np.float64)
    if act == "gelu":
        return 0.5 * erfc(-z / np.sqrt(2)) + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    if act == "gelu_tanh":
        s = expit(_A * (z + _B * z ** 3))
        return s + z * s * (1 - s) * _A * (1 + 3 * _B * z ** 2)
    if act == "silu":
        s = expit(z)
        return s + z * s * (1 - s)
    return np.ones_like(z)


def value_bound(z, act):
    """Of act(z), z an fp32 number, in fp32: an exponential of an argument A that is rounded a few times (A at most
    z^2 + 2 |z| here: relative error 2^-22 A), a fit to 8e-7, and a few operations on z itself (2^-22 |z|)."""
    if act in ("none", "relu"):
        return np.zeros_like(z)
    return np.abs(value(z, act)) * (2e-6 + 2.0 ** -22 * (z * z + 2 * np.abs(z))) + 2.0 ** -22 * np.abs(z)


def slope_bound(z, act):
    """Slopes are sums of two terms of size 1.2 at most, each within a few 2^-22 and the exponential's error."""
    return np.zeros_like(z) if act in ("none", "relu") else np.full_like(z, 2e-6)


# half a step of a type relative to a value, and in its subnormal range
ROUNDING = {"f32": (2.0 ** -24, 2.0 ** -149), "f16": (2.0 ** -11, 2.0 ** -25), "bf16": (2.0 ** -8, 2.0 ** -133)}
