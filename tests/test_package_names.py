"""The package's functions are those of ``api``, looked up at every use: a program that replaces one there is heard.  CPU only."""
import pytest

import paper_2308_10037_b200 as package
from paper_2308_10037_b200 import api


@pytest.mark.parametrize("name", package._FROM_API)
def test_a_replaced_function_is_found_through_the_package(monkeypatch, name):
    assert getattr(package, name) is getattr(api, name)
    other = object()
    monkeypatch.setattr(api, name, other)
    assert getattr(package, name) is other
