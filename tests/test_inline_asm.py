"""What the inline assembly uses and changes has to be known to the compiler (read from the sources; no GPU)."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _statements():
    for path in sorted(glob.glob(os.path.join(ROOT, "paper_2401_04044_amd", "csrc", "*"))):
        if path.endswith((".hip", ".h")):
            for m in re.finditer(r"\basm\s+volatile\s*\((.*?)\);", open(path).read(), re.S):
                yield os.path.basename(path), m.group(1)


def test_m0_is_written_by_the_compiler_alone():
    """m0 is a reserved register: a statement that writes it cannot say so, one that needs a value in it takes it as an operand."""
    for name, text in _statements():
        assert not re.search(r"s_\w+\s+m0\s*,", text), (name, text)
        if re.search(r"buffer_load\S*.*\blds\b", text):
            assert '"{m0}"' in text, (name, text)


def test_statements_that_touch_memory_or_order_it_say_so():
    for name, text in _statements():
        if re.search(r"\b(s_barrier|s_waitcnt|buffer_load|global_load|ds_)", text):
            assert '"memory"' in text.rsplit(":", 1)[1], (name, text)
