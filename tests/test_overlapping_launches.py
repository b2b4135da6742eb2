"""Kernels that may start before those that write what they read have ended."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_18954_gb300", "csrc")


def test_what_a_call_writes_is_not_read_as_constant():
    """Where kernels wait for those before them (after_previous), the non-coherent loads, for data that is constant while a kernel
    runs, take none of the call's own arrays."""
    for name in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, name)).read()
        if name.endswith(".cu") and "after_previous()" in text:
            for use in re.findall(r"(?:__ldg|ld\.global\.nc)[^;]*;", text):
                # (the embedding's table and gradient rows are inputs)
                assert name == "gpo_embed.cu" and "row + at(" in use, (name, use)
