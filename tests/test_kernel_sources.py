"""Rules that every kernel has to keep for the ones around it, read off the sources: a mistake here would hang the GPU, so it is not
left to a run to find."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2301_01333_b200", "csrc")
SOURCES = sorted(f for f in os.listdir(CSRC) if f.endswith(".cu"))


def code_of(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name", SOURCES)
def test_tensor_memory_is_taken_before_the_next_kernel_may_start(name):
    """From the moment a kernel lets its successor start, the successor's blocks can take tensor memory and then wait for this
    kernel's end; one warp of a block takes the columns, so a barrier of the block has to lie in between."""
    code = code_of(name)
    for take in re.finditer(r"\btmem_alloc2?\(smem", code):
        rest = code[take.end():]
        go = re.search(r"griddepcontrol\.launch_dependents|wait_for_predecessor\(\)", rest)
        if go:
            assert re.search(r"__syncthreads\(\)|cluster_sync_all\(\)", rest[:go.start()]), f"{name}: the next kernel may start too early"


def test_the_rule_is_looked_for_where_it_matters():
    taking = [n for n in SOURCES if re.search(r"\btmem_alloc2?\(smem", code_of(n))]
    letting = [n for n in taking if "launch_dependents" in code_of(n) or "wait_for_predecessor" in code_of(n)]
    assert "kernels_attn_prompt.cu" in letting and "kernels_gemm_tc.cu" in letting and len(letting) >= 8


@pytest.mark.parametrize("name", [n for n in SOURCES if "launch_following(" in code_of(n)])
def test_nothing_is_read_before_the_kernel_has_waited(name):
    """Kernels that are started while the one before them still runs read its results, and those of the ones before it, only behind
    griddepcontrol.wait; nothing else promises that they are there."""
    code = code_of(name)
    kernels = re.split(r"__global__ void", code)[1:]
    assert kernels
    for k in kernels:
        wait = re.search(r"griddepcontrol\.wait|wait_for_predecessor\(\)", k)
        assert wait, "a kernel that does not wait"
        ahead = k[k.index("{"):wait.start()]
        found = re.search(r"length_of|blocks_of|all_blocks|sequence_at|seq_of|\bp\.(\w+)\[|p\.ws|->|ld\.global|cp\.async", ahead)
        assert not found, f"{name}: '{found.group(0)}' ahead of the wait"


@pytest.mark.parametrize("name", [n for n in SOURCES if "setmaxnreg.inc" in code_of(n)])
def test_registers_are_only_taken_where_the_launch_has_them(name):
    """setmaxnreg.inc beyond the registers a block was launched with waits for good, and how many those are is the compiler's
    decision: the host has to ask before it launches, and the shares have to add up."""
    code = code_of(name)
    assert re.search(r"numRegs", code) and re.search(r"static_assert\([^;]*REGS", code), f"{name} trusts the compiler's register count"


@pytest.mark.parametrize("name", [n for n in SOURCES if re.search(r"\bmma_ts\(", code_of(n))])
def test_scores_wait_for_the_product_that_reads_what_they_overwrite(name):
    """Only products into one accumulator, of one shape, are promised to run in the order they were issued in.  Scores that are written over
    probabilities therefore wait until the product that reads these is complete: a wait lies between the last such product and the
    next scores, and one ahead of the first scores of an item where the item before may still be read."""
    code = code_of(name)
    last = [m.start() for m in re.finditer(r"\bmma_ts\(", code)][-1]
    nxt = re.search(r"(?<!auto )\bscores\(", code[last:])
    assert nxt, "scores are issued behind the products with probabilities"
    assert re.search(r"p_is_read\(\)|mma_wait\(o_full", code[last:last + nxt.start()]), f"{name}: nothing keeps the next scores behind the product that reads"
    begin = re.search(r"auto begin = .*?scores\(", code, re.S)
    assert not begin or "p_is_read()" in begin.group(0), f"{name}: the first scores of an item"


def test_every_stretch_of_the_chunk_attention_has_a_block_to_write():
    """The joining kernel reads a piece of every CTA between an item's first and last: a stretch that lay inside one block of keys would leave its
    piece unwritten.  The CTAs at work are as many as get CK_LEAST units each, whatever the total comes to."""
    code = code_of("kernels_attn_chunk.cu")
    value = {k: int(v) for k, v in re.findall(r"\b(CK_LEAST|CK_START|CK_BLOCK|CK_TWIN_BLOCK) = (\d+)", code)}
    assert re.search(r"fill = quotient\(total, CK_LEAST\);", code) and re.search(r"static_assert\(CK_LEAST >= CK_BLOCK", code)
    for total in range(value["CK_START"] + min(value["CK_BLOCK"], value["CK_TWIN_BLOCK"]), 5000):
        for ctas in (1, 2, 7, 148):
            working = min(max(total // value["CK_LEAST"], 1), ctas)
            assert total // working >= value["CK_LEAST"] >= max(value["CK_BLOCK"], value["CK_TWIN_BLOCK"])
