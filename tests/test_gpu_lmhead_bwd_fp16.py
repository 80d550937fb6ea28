"""Every test of the LM head's gradient once more with dz of one fp16 above 128 rows (the library by itself takes two bf16 terms for sizes like theirs) (GPU)."""
import pytest

from paper_2604_04215_amd import binding as dlm
from test_gpu_lmhead_bwd import *  # noqa: F401,F403  (the tests)


@pytest.fixture(autouse=True)
def few():
    dlm.set_option("lmhead_bwd_few", 128)
    yield
    dlm.set_option("lmhead_bwd_few", 0)
