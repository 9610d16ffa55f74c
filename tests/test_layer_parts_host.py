"""That the checks of FP32 layers tell a product with all its parts from one without, on the CPU: the parts and their six products in 64 bits."""
import itertools

import pytest
import torch

import test_gpu_linear_f32 as f32

SIX = [(2, 0), (0, 2), (1, 1), (1, 0), (0, 1), (0, 0)]
NAMES = {"p1 q2": (0, 1), "p2 q1": (1, 0), "p2 q2": (1, 1), "p1 q3": (0, 2), "p3 q1": (2, 0)}


def parts(x):
    out, rest = [], x
    for _ in range(3):
        p = rest.to(torch.bfloat16).float()
        out.append(p.double())
        rest = rest - p
    assert not rest.any()      # 24 bits: three parts hold them all
    return out


def product(A, B, pairs):
    p, q = parts(A), parts(B)
    return sum(p[i] @ q[j].t() for i, j in pairs)


@pytest.mark.parametrize("name", sorted(f32.PARTS))
def test_each_planted_product_needs_its_parts(name):
    A, B, want = f32.planted(name, 20, 12, 40, 6, device="cpu")
    assert torch.equal(product(A, B, SIX), want.double()) and torch.equal(A.double() @ B.double().t(), want.double())
    assert (product(A, B, [pair for pair in SIX if pair != NAMES[name]]) != want.double()).all()


def test_the_size_of_the_error_shows_what_is_missing():
    """In units of 2^-24 of the root of the sum of squares, where the check takes 32: all six products are below one, without any third part, or any of the products that
    hold one, it is more; without p2 q2 the planted cases tell."""
    gen = torch.Generator().manual_seed(1)
    A, B = torch.randn(100, 512, generator=gen), torch.randn(80, 512, generator=gen)
    want, size = A.double() @ B.double().t(), ((A.double() ** 2) @ (B.double() ** 2).t()).sum().sqrt()

    def units(pairs):
        return float((product(A, B, pairs) - want).square().sum().sqrt() / size * 2 ** 24)

    assert units(SIX) < 1
    for missing in [m for n in (1, 2, 3) for m in itertools.combinations([(2, 0), (0, 2), (1, 0), (0, 1)], n)]:
        assert units([pair for pair in SIX if pair not in missing]) > 32, missing
