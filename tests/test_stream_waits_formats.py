"""The stream pass over 4-bit pools and with windows keeps the rules of its older variants, in the assembly that its sources give (no GPU): the loops that
send hidden stores off do not wait for them, dynamic LDS begins aligned, nothing is spilled to memory."""
import os
import re
import subprocess

import pytest

from paper_2602_11530_amd import build as pkv_build
from test_stream_waits import CSRC, loops_with_hidden_stores

SOURCES = {"attn_stream_fp4": 6, "attn_stream_span": 9, "attn_stream_span_short": 12}   # and how many variants


@pytest.fixture(scope="module", params=SOURCES)
def assembly(request, tmp_path_factory):
    asm = str(tmp_path_factory.mktemp("asm") / "out.s")
    flags = [f for f in pkv_build.FLAGS if f not in ("-fPIC", "-shared")]
    subprocess.check_call([pkv_build.HIPCC, *flags, "--cuda-device-only", "-S", os.path.join(CSRC, request.param + ".hip"), "-o", asm],
                          stderr=subprocess.DEVNULL)
    return SOURCES[request.param], open(asm).read()


def test_store_loops_do_not_wait_for_their_stores(assembly):
    variants, text = assembly
    kernels = re.findall(r"^(_ZN\S*attn_stream_kernel\S*):(.*?)^\.Lfunc_end", text, re.S | re.M)
    assert len(kernels) == variants
    for name, body in kernels:
        found = list(loops_with_hidden_stores(body.split("\n")))
        assert len(found) >= 5, (name, found)
        # no wait at all: no register of a load that may be under way is taken over there
        assert not any(waits for _, _, waits in found), (name, found)


def test_lds_begins_aligned(assembly):
    variants, text = assembly
    sizes = re.findall(r"\.amdhsa_group_segment_fixed_size (\d+)", text)
    assert len(sizes) == variants and all(int(s) % 16 == 0 for s in sizes), sizes


def test_nothing_is_spilled_to_memory(assembly):
    variants, text = assembly
    private = re.findall(r"\.amdhsa_private_segment_fixed_size (\d+)", text)
    assert private == ["0"] * variants
