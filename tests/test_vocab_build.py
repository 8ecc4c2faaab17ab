"""Build invariants of the kernels on the vocabulary's matrix and logits, from the compiler's own report: no scratch memory where rows are
in registers, waves as the launches count on, no packed fp32 arithmetic, and main loops as they are meant."""
import os
import re
import subprocess
import tempfile

import pytest

from paper_2603_16428_amd import build as B


@pytest.fixture(scope="module")
def report():
    """({kernel: its resources}, the assembly) of all sources, compiled at the same time."""
    with tempfile.TemporaryDirectory() as d:
        started = []
        for k, source in enumerate(B.VOCAB_SOURCES):
            out = os.path.join(d, f"{k}.s")
            cmd = [B.HIPCC] + [f for f in B.FLAGS if f != "-shared"] + ["-S", "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", source, "-o", out]
            started.append((out, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)))
        kernels, text = {}, ""
        for out, p in started:
            err = p.communicate()[1]
            assert p.returncode == 0, err[-2000:]
            for part in re.split(r"Function Name: ", err)[1:]:
                kernels[part.split()[0]] = {k: int(re.search(re.escape(k) + r"[^:]*: (\d+)", part).group(1))
                                            for k in ("VGPRs", "ScratchSize", "Occupancy", "LDS Size")}
            text += open(out).read()
        return kernels, text


def _of(kernels, name):
    found = {n: use for n, use in kernels.items() if re.search(r"\d" + name + r"(I|E)", n)}
    assert found, name
    return found


def test_no_scratch_memory(report):
    kernels, _ = report
    for name in ("embedding_kernel", "embedding_sort_kernel", "embedding_merge_tiles_kernel", "embedding_merge_kernel", "embedding_sum_kernel", "embedding_join_kernel",
                 "mxfp4_quantize_kernel", "mxfp4_dequantize_kernel", "mxfp4_few_kernel", "mxfp4_many_kernel", "sample_parts_kernel"):
        for n, use in _of(kernels, name).items():
            assert use["ScratchSize"] == 0, (n, use)


def test_waves(report):
    """Two workgroups of the product's kernel for few rows a CU, one of that for many (eight waves, or four in the smaller tile), one of a
    row's sampling."""
    kernels, _ = report
    for n, use in _of(kernels, "mxfp4_few_kernel").items():
        assert use["Occupancy"] >= 2 and use["LDS Size"] <= 80 * 1024, (n, use)
    for n, use in _of(kernels, "mxfp4_many_kernel").items():
        assert use["Occupancy"] >= (2 if n.count("Li256ELi8E") else 1), (n, use)
    for n, use in _of(kernels, "sample_row_kernel").items():
        assert use["Occupancy"] >= 4 and use["LDS Size"] <= 160 * 1024, (n, use)


def test_no_packed_fp32(report):
    assert not re.search(r"v_pk_(add|mul|fma)_f32", report[1])


def test_products_wait_for_their_own_step_alone(report):
    """In the main loop for few rows the next step's loads are on the way while the current one's products run: no wait for all of them."""
    _, text = report
    for name in re.findall(r"^(_ZN3lce16mxfp4_few_kernel\S+):", text, re.M):
        body = text[text.index(name + ":"):]
        body = body[:body.index(".Lfunc_end")]
        # The loop is the stretch from the first product on that holds both products and wide loads.
        blocks = [b for b in re.split(r"^\.LBB\w+:", body, flags=re.M) if b.count("v_mfma_scale") >= 4 and "buffer_load_dwordx4" in b]
        assert blocks, name
        loop = max(blocks, key=lambda b: b.count("buffer_load_dwordx4"))
        first = loop.index("v_mfma_scale")
        waits = [int(n) for n in re.findall(r"vmcnt\((\d+)\)", loop[:first])]
        assert waits and max(waits) > 0, (name, waits)


def test_neither_half_of_the_loop_waits_for_all_loads(report):
    """The same for every wait in both halves of the loop (two steps, each with the loads of the one after it); only the last, shorter step, behind
    it, waits for all that is on the way."""
    _, text = report
    names = re.findall(r"^(_ZN3lce16mxfp4_few_kernel\S+):", text, re.M)
    assert names
    for name in names:
        body = text[text.index(name + ":"):]
        body = body[:body.index(".Lfunc_end")]
        blocks = [b for b in re.split(r"^\.LBB\w+:", body, flags=re.M) if b.count("v_mfma_scale") >= 4 and "buffer_load_dwordx4" in b]
        waits = [[int(n) for n in re.findall(r"vmcnt\((\d+)\)", b)] for b in blocks]
        assert len(blocks) == 3 and all(w and min(w) > 0 for w in waits[:2]), (name, waits)


def test_a_row_of_logits_spills_no_more_than_is_known(report):
    """The row's kernel of sampling has all its paths in 128 registers of 1024 threads, and spills: 200 bytes a lane in 16 bits, 268 in fp32 (up to
    2^18 logits), 300 at most."""
    kernels, _ = report
    for n, use in _of(kernels, "sample_row_kernel").items():
        usual = "Li1ELNS_6RowEndE1E" in n
        assert use["ScratchSize"] <= ((272 if "kernelIfLi" in n else 204) if usual else 304), (n, use)
