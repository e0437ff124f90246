"""The binding of the products, decaying states and group norms on the CPU: what does not need a device."""
import paper_2609_31938_b200 as ccv


def test_status_words_refuse_what_is_none():
    assert ccv.lib.ccv3d_linear_status_word(None) == ccv.ERR_INVALID_ARG
    assert ccv.ccv3d_take_status(None)[0] == ccv.ERR_INVALID_ARG
    assert ccv.ccv3d_take_status(6)[0] == ccv.ERR_ALIGNMENT
