"""Scores where the number of rows, with their length, decides which kernel a row gets, against the definition in 64 bits (tolerances as in
test_gpu_policy_scores.py)."""
import pytest

from test_gpu_policy_scores import _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,V,k,dtype,mask", [
    # a wavefront for each of many rows of up to 8192 entries
    (2048, 2049, 0, "float32", None), (2100, 5001, 5, "bfloat16", "rows"), (2050, 8191, 20, "float16", "shared"), (2100, 4097, 64, "float32", "rows"),
    # four wavefronts for a row of fewer, or of longer rows than there are compute units
    (2047, 2049, 0, "bfloat16", "rows"), (300, 8193, 0, "float32", None), (257, 20001, 5, "float16", "rows"), (260, 9001, 64, "bfloat16", "shared"),
    # sixteen for a long row; too many rows to be cut into pieces
    (65, 40001, 0, "bfloat16", "rows"), (70, 33001, 20, "float32", None), (256, 8193, 64, "float16", "rows"),
    # pieces of few long rows, as long as a work-group loads at once or longer
    (64, 32769, 20, "float32", "rows"), (3, 32770, 64, "bfloat16", None), (1, 600001, 20, "float16", "shared"),
    # short rows held by few lanes: more alternatives where rows are many
    (8191, 100, 17, "bfloat16", "rows"), (8192, 100, 17, "bfloat16", "rows"), (8200, 127, 32, "float32", None), (8192, 31, 32, "float16", "shared"), (8200, 7, 33, "float32", "rows"),
    # rows of 129 to 512 entries held by a wavefront, with few alternatives
    (500, 129, 3, "float32", "rows"), (33, 511, 3, "bfloat16", None), (2100, 512, 4, "float16", "rows")])
def test_against_the_definition(N, V, k, dtype, mask):
    _check(*_inputs(N, V, dtype, mask), k=k, scale=0.9)
