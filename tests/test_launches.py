"""The launches that the library makes, checked without a GPU (tests/launches.py)."""
import pytest

from tests import launches


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    return launches.build(tmp_path_factory.mktemp("recorder"))


@pytest.mark.parametrize("check", ["work_lists_of_one_type", "work_lists_of_the_same_memory_in_another_type"])
def test_orthogonalize(recorder, check):
    launches.run(recorder, check)


def test_layer_norm_rows(recorder):
    """Any number of rows that the call takes, in launches that HIP takes."""
    launches.run(recorder, "layer_norm_rows")
