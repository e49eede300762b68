"""Direct loads into LDS take their address from M0, a register that the compiler may write between any two statements: every such load in the
kernels' sources sets it in its own statement (no GPU)."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_08923_amd", "csrc")


def test_every_load_sets_its_address():
    seen = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for asm in re.findall(r'asm\s+volatile\s*\(((?:\s*"(?:[^"\\]|\\.)*")+)', text):
            for at in re.finditer(r"buffer_load[^\"\n]*?\blds\b", asm):
                seen += 1
                assert "s_mov_b32 m0" in asm[:at.start()], (os.path.basename(path), asm)
    assert seen >= 5
