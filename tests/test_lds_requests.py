"""The attention's tiles go from memory to LDS by instructions written by hand, whose place in LDS is in m0, a register that the compiler
takes for its own.  In the library as it was built it uses it for nothing else in these kernels: m0 is written right before such
requests alone, and every wave waits for its own before each barrier that hands a tile over."""
import os
import re

import pytest

from paper_2210_15458_amd import binding
from test_reads_in_flight import OBJDUMP, kernels


@pytest.mark.skipif(not os.path.exists(OBJDUMP) or not os.path.exists(binding.LIB_PATH), reason="no disassembler, or no library")
def test_m0_is_the_requests_own(tmp_path):
    found = kernels(tmp_path, "attend_tiles_kernel")
    found = {name: code for name, code in found.items() if any("global_load_lds" in text for _, text, _ in code)}
    assert len(found) == 18                       # (three widths, three forms of rows, prompts shared and ragged)
    for name, code in found.items():
        texts = [text for _, text, _ in code]
        requests = [i for i, text in enumerate(texts) if text.startswith("global_load_lds_dwordx4")]
        for i, text in enumerate(texts):
            if re.search(r"\bm0\b", text):
                assert re.match(r"s_mov_b32 m0, s\d+$", text), (name, text)
                assert texts[i + 1].startswith("s_nop") and i + 2 in requests, (name, texts[i:i + 3])
        for i in requests:                        # each is behind such a write, or behind another of the same
            j = i
            while texts[j - 1].startswith("global_load_lds_dwordx4"):
                j -= 1
            assert texts[j - 1].startswith("s_nop") and texts[j - 2].startswith("s_mov_b32 m0"), (name, texts[j - 3:i + 1])
        waits = [i for i, text in enumerate(texts) if text.startswith("s_waitcnt") and "vmcnt(0)" in text and "lgkmcnt(0)" in text and texts[i + 1].startswith("s_barrier")]
        assert len(waits) == 3, name              # the first tile's, and one in each half of the loop over pairs of tiles
