"""The products that the GPU tests run reach every kernel of csrc/i8_choice.h, the linear layers too."""
from __future__ import annotations

import pytest

from layers_sizes import PRODUCTS, SHORT, SKINNY_LINEAR
from test_layers_choice import choice  # noqa: F401  (a fixture)


@pytest.mark.parametrize("m,n,k,kernel", PRODUCTS)
def test_kernel(choice, m, n, k, kernel):  # noqa: F811
    assert choice.product(m, n, k) == kernel


def test_every_kernel_is_reached(choice):  # noqa: F811
    assert {p[3] for p in PRODUCTS} == set(range(7))
    plain = {k for m, n, k_, k in PRODUCTS if not choice.skinny(m, n, k_) and not choice.tile(m, n, k_)}
    assert plain == set(range(7)) and SHORT in plain


def test_linear_layers_up_to_the_limit_of_lds(choice):  # noqa: F811
    padded = [(m, n, -(-k // 16) * 16) for m, n, k in SKINNY_LINEAR]
    assert all(choice.skinny(*s) for s in padded)
    assert max(m * (k + 16) for m, _, k in padded) == 64 << 10
