"""sbp_matmul8_set_form without a GPU: which forms there are."""
import pytest

import paper_2110_15032_b200 as sbp


def test_forms_that_do_not_exist_are_refused():
    from paper_2110_15032_b200.build import build
    build()
    try:
        for columns, splits, exchanged in ((256, 1, False), (128, 8, True), (16, 4, False), (0, 1, False)):
            sbp.sbp_matmul8_set_form(columns, splits, exchanged)
        for columns, splits, exchanged in ((256, 2, False), (256, 1, True), (100, 1, False), (-128, 1, False), (128, 3, False), (128, 16, False), (64, 0, False)):
            with pytest.raises(sbp.SbpError) as e:
                sbp.sbp_matmul8_set_form(columns, splits, exchanged)
            assert e.value.name == "SBP_ERR_INVALID_ARG"
        assert sbp.sbp_matmul8_form_launches(99, 1, False, True, True) == 0
    finally:
        sbp.sbp_matmul8_set_form()
