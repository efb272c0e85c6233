"""Blocks decide as one whether an earlier error stops them.

Calls on several streams may share a status word, so it can change while a kernel's threads look at it.  Where threads of a block
meet at barriers that count them, or take parts in a pipeline, a thread must not read the word for itself: those that went on would
wait for those that left.  ``block_sees_error`` asks once for all of them; ``warp_sees_error`` asks for a warp, and warps that meet
at a named barrier agree on the answer.  (The barrier of a whole block does not count threads that have left.)"""
import os
import re

import pytest

import paper_2210_00129_b200 as sbp

CSRC = os.path.join(os.path.dirname(sbp.__file__), "csrc")
READ = re.compile(r"\*[^;,&|]*\bstatus_word\)?\s*[!=]=\s*0")          # the word itself against zero, not its address


def reads(name):
    with open(os.path.join(CSRC, name)) as f:
        return READ.findall(re.sub(r"//[^\n]*", "", f.read()))


@pytest.mark.parametrize("name", ["block_norm.cu", "embedding.cu", "orthogonalize.cu", "attention_bwd.cu", "split_products.cu",
                                  "tc_backward.cu", "tc_forward.cu"])
def test_no_thread_reads_the_word_for_itself(name):
    assert not reads(name)


@pytest.mark.parametrize("line", ["if (p.status_word != nullptr && *p.status_word != 0) return;",
                                  "skip = *reinterpret_cast<volatile int32_t*>(status_word) != 0;"])
def test_the_pattern_finds_reads(line):
    assert READ.findall(line) and not READ.findall("if (p.status_word != nullptr) f(*p.x, p.status_word);")
