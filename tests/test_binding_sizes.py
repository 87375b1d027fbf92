"""Sizes that pass 32 bits are Python errors in the extension, never taken modulo 2^32.  No GPU is needed."""
import pytest

from test_binding_errors import run

CALLS = {
    "spmm_csr": "native.spmm_csr({x}, {y}, {y}, None, None, None, t, t, None)",
    "sddmm_csr": "native.sddmm_csr({y}, {y}, {x}, None, None, None, t, t, None, None)",
    "coo_to_csr_rowptr": "native.coo_to_csr_rowptr({x}, None, None, None, None)",
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_sizes_beyond_32_bits(name):
    body = """
with FakeTensorMode():
    t = torch.zeros(0, 0, device="cuda")
class Stream:
    cuda_stream = 0
"""
    for x in (2 ** 31, 2 ** 32, 2 ** 32 + 1, -2 ** 31 - 1, 2 ** 70):
        call = CALLS[name].format(x=x, y=0).replace("None)", "Stream)")
        body += f"try:\n    {call}\n    print('taken')\nexcept (OverflowError, ValueError) as e:\n    print('refused' if '32 bits' in str(e) or 'too' in str(e) else e)\n"
    assert run(body) == ["refused"] * 5
