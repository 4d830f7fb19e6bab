"""After a call that CUDA refused, the process goes on as if it had not been made."""

import pytest
import torch

from paper_2602_01901_b200 import binding as qc
from paper_2602_01901_b200 import quant

pytestmark = pytest.mark.gpu


def calls():
    from test_quant_cpu import OK_TABLE, SHAPE, attend_args

    t, s, no = qc.qc_table(**OK_TABLE), qc.qc_quant_shape(**SHAPE), 4096      # a device that is not there
    return {
        "reset": lambda: qc.qc_table_reset(no, 0, t), "extend": lambda: qc.qc_table_extend(no, 0, t, 1, 0, 0, 1, 64, 64),
        "trim": lambda: qc.qc_table_trim(no, 0, t, 1, 0, 0), "append": lambda: qc.qc_quant_append(no, 0, s, 1, 64, 64, 256, 64, 256, 64, 64),
        "read": lambda: qc.qc_quant_read(no, 0, s, 1, 64, 64, 64, 64, 64), "attend": lambda: qc.qc_quant_attend(no, 0, attend_args()),
    }


@pytest.mark.parametrize("name", ["reset", "extend", "trim", "append", "read", "attend"])
def test_a_device_that_is_not_there_leaves_no_error_behind(name):
    x = torch.arange(4.0, device="cuda")
    with pytest.raises(qc.QcError) as e:
        calls()[name]()
    assert e.value.status == qc.QC_ERR_CUDA and torch.cuda.current_device() == 0
    assert (x + 1).tolist() == [1.0, 2.0, 3.0, 4.0]
    table = quant.PageTable.empty(2, 2, 16, 4)
    assert quant.table_extend(table)[1].tolist() == [0, 16]
