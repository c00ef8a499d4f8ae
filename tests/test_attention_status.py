"""The status of the attention kernels on a device: one reading takes in and clears the
words of all of them, so that a later one tells of later calls alone."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def read(tmp_path_factory):
    from paper_2607_19368_gb300 import build
    exe = str(tmp_path_factory.mktemp("status") / "attention_status")
    subprocess.run([build.nvcc()] + build.ARCH + build.NVCC_FLAGS +
                   [os.path.join(HERE, "host", "attention_status.cu"), "-o", exe], check=True)

    def ask(prefill, decode):
        out = subprocess.run([exe], input=f"{prefill} {decode}", capture_output=True, text=True,
                             check=True).stdout
        return [int(x) for x in out.split()]

    return ask


@pytest.mark.parametrize("prefill,decode,first", [(0, 0, 0), (5, 0, 5), (0, 5, 5), (5, 5, 5),
                                                  (5, 6, 5)])
def test_every_word_is_read_and_cleared(read, prefill, decode, first):
    assert read(prefill, decode) == [first, 0, 0]
