"""The bound that the layer norm's kernels are held to where a row's mean is large
against its deviations (test_gpu_layer_norm.py), on forms of it in fp32 on the
CPU: it lets through the one that takes the mean's own error off, and none that
loses the deviations."""
import pytest
import torch

from tests.test_gpu_layer_norm import D, EPS, LARGE_MEANS, about_a_large_mean

COLS = 4096


def rows(mean, size):
    g = torch.Generator().manual_seed(1)
    h = torch.randn(6, COLS, generator=g) * size + mean
    return h, 1 + 0.2 * torch.randn(COLS, generator=g), 0.1 * torch.randn(COLS, generator=g)


def total(x):
    """Row sums as the kernels form them: a thread's 16 values one after the other, then the threads' in pairs."""
    s = x.view(x.shape[0], -1, 16)
    run = s[:, :, 0].clone()
    for i in range(1, 16):
        run = run + s[:, :, i]
    while run.shape[1] > 1:
        run = run[:, ::2] + run[:, 1::2]
    return run


def corrected(h, w, b):
    mean = total(h) / COLS
    d = h - mean
    rest = total(d) / COLS
    var = (total(d * d) / COLS - rest * rest).clamp_min(0)
    rstd = 1 / (var + EPS).sqrt()
    return (mean + rest)[:, 0], rstd[:, 0], (d - rest) * rstd * w + b


def two_pass(h, w, b):
    mean = total(h) / COLS
    d = h - mean
    rstd = 1 / (total(d * d) / COLS + EPS).sqrt()
    return mean[:, 0], rstd[:, 0], d * rstd * w + b


def one_pass(h, w, b):
    mean = total(h) / COLS
    var = (total(h * h) / COLS - mean * mean).clamp_min(0)
    rstd = 1 / (var + EPS).sqrt()
    return mean[:, 0], rstd[:, 0], (h - mean) * rstd * w + b


def nothing(h, w, b):
    return h.new_zeros(len(h)), h.new_zeros(len(h)), torch.zeros_like(h)


def holds(form, mean, size):
    h, w, b = rows(mean, size)
    want, tol = about_a_large_mean(h, w, b)
    return [bool(((g.double() - t).abs() <= e).all()) for g, t, e in zip(form(h, w, b), want, tol)]


@pytest.mark.parametrize("mean,size", LARGE_MEANS)
def test_the_corrected_form_holds(mean, size):
    assert holds(corrected, mean, size) == [True, True, True]


@pytest.mark.parametrize("mean,size", [c for c in LARGE_MEANS if 0 < c[1] < abs(c[0])])
def test_the_others_do_not(mean, size):
    """y is what they lose; one pass loses rstd as well where the mean is 2^12 times the deviations."""
    assert not holds(two_pass, mean, size)[2]
    assert not holds(one_pass, mean, size)[2]
    assert holds(nothing, mean, size) == [False, False, False]
    if abs(mean) > 4096 * size:
        assert not holds(one_pass, mean, size)[1]
