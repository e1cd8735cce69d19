"""The kernels of prompts and of pools with a scale for each block and KV head, in the assembly that their sources give (no GPU)."""
import os
import re
import subprocess

import pytest

from paper_2602_11530_amd import build as pkv_build
from test_stream_waits import CSRC, loops_with_hidden_stores

SOURCES = {"prompt_attn": 24, "attn_stream_blk": 7, "kv_append_blk": 12}   # and how many kernels


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    flags = [f for f in pkv_build.FLAGS if f not in ("-fPIC", "-shared")]
    where, running = tmp_path_factory.mktemp("asm"), []
    for source in SOURCES:
        running.append(subprocess.Popen([pkv_build.HIPCC, *flags, "--cuda-device-only", "-S", os.path.join(CSRC, source + ".hip"), "-o",
                                         str(where / (source + ".s"))], stderr=subprocess.DEVNULL))
    assert all(p.wait() == 0 for p in running)
    return {source: (where / (source + ".s")).read_text() for source in SOURCES}


def kernels(text, name):
    return re.findall(rf"^(_ZN\S*{name}\S*):(.*?)^\.Lfunc_end", text, re.S | re.M)


@pytest.mark.parametrize("source", SOURCES)
def test_nothing_is_spilled_to_memory(assembly, source):
    """Or next to nothing, once before a loop over keys and once behind it."""
    sizes = [int(n) for n in re.findall(r"\.amdhsa_private_segment_fixed_size (\d+)", assembly[source])]
    assert len(sizes) == SOURCES[source]
    for n, (name, body) in zip(sizes, kernels(assembly[source], "kernel"), strict=True):
        lines = body.split("\n")
        scratch, products = ([i for i, x in enumerate(lines) if word in x] for word in ("scratch_", "v_mfma"))
        assert not scratch or (n <= 8 and "prompt_attn_kernel" in name), (name, n)
        assert not any(products[0] <= i <= products[-1] for i in scratch), name


def test_stream_pass_keeps_the_rules_of_its_other_variants(assembly):
    text = assembly["attn_stream_blk"]
    found = kernels(text, "attn_stream_kernel")
    assert len(found) == SOURCES["attn_stream_blk"]
    for name, body in found:
        loops = list(loops_with_hidden_stores(body.split("\n")))
        assert len(loops) >= 5 and not any(waits for _, _, waits in loops), (name, loops)
    sizes = re.findall(r"\.amdhsa_group_segment_fixed_size (\d+)", text)
    assert all(int(s) % 16 == 0 for s in sizes), sizes


def test_loads_straight_to_lds(assembly):
    """The compiler does not know that those loads use M0 nor what they write: M0 is set right before each, nothing else in the kernel has a use for it,
    and what a wavefront loaded is waited for before others read it: where four share it as it is, at the next barrier."""
    found = 0
    for name, body in kernels(assembly["prompt_attn"], "prompt_attn_kernel"):
        lines = [x.split(";")[0].strip() for x in body.split("\n")]
        lines = [x for x in lines if x]
        loads = [i for i, x in enumerate(lines) if x.startswith("buffer_load") and x.endswith("lds")]
        bf16 = re.search(r"ILi\d+ELi0ELi", name)
        alone = "Lb1E" in name
        assert bool(loads) == bool(bf16 or "ILi256E" in name and not alone), name
        found += len(loads) > 0
        for i in loads:
            assert lines[i - 2].startswith("s_mov_b32 m0,") and lines[i - 1] == "s_nop 0", lines[i - 3:i + 1]
        assert sum(bool(re.search(r"\bm0\b", x)) for x in lines) == len(loads)
        for i in loads if bf16 and not alone else ():
            rest = lines[i + 1:]
            barrier = next((k for k, x in enumerate(rest) if x.startswith("s_barrier")), None)
            if barrier is not None:
                assert any(re.match(r"s_waitcnt.*vmcnt\(0\)", x) for x in rest[:barrier]), (name, i)
    assert found == 9
