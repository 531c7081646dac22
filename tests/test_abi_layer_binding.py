"""Refusals of the Python functions that need no GPU."""
import pytest
import torch

from paper_2412_01034_b200 import api, build


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def test_check_workspace_refuses_what_is_no_workspace():
    with pytest.raises(ValueError):
        api.check_workspace(torch.zeros(64, dtype=torch.uint8))
