"""What `frequencies` refuses beside what test_attention_host.py has."""
import pytest


@pytest.mark.parametrize("base,scaling", [(1e300, {"kind": "base", "factor": 1e30}), (1e4, {"kind": "base", "factor": 1e306})])
def test_a_base_that_overflows_is_refused(base, scaling):
    from paper_2608_21614_b200 import binding as B, rotary
    with pytest.raises(B.SaemError) as e:
        rotary.Rotary(64, base=base, scaling=scaling, device="cpu")
    assert e.value.code == B.SAEM_ERR_INVALID_ARG
