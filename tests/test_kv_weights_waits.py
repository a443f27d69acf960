"""Waits of the kernels of the attention weights by token, read from their source: what an expired one, or one that comes too late, would spoil."""
import re
from pathlib import Path

CSRC = Path(__file__).resolve().parent.parent / "paper_2011_09398_b200" / "csrc"


def test_producers_of_keys_publish_nothing_behind_a_wait_that_gave_up():
    """Every wait of the loop is followed by a meeting of all its warps that they leave from together, before anything is written to
    the operands' place or announced, and before the next tile's wait could forget the result."""
    text = (CSRC / "kv_weights_prompt.cu").read_text()
    loop = text[text.index("tile.begin(p, sh, count);\n        for (uint32_t n = 0"):text.index("// ---- the products")]
    steps = {"wait": r"ok = wait_bounded\(", "meet": r"ok = half_sync_and\(1, ok\);[^\n]*\n\s*if \(!ok\) break;", "publish": r"sh\.info\[|decode\(|mbar_arrive\(&sh\.bars\[BAR_(?:STREAM|STAY)_FULL"}
    found = sorted((m.start(), kind) for kind, pattern in steps.items() for m in re.finditer(pattern, loop))
    kinds = [kind for _, kind in found]
    assert kinds.count("wait") == 3 and kinds.count("meet") >= 2 and kinds.count("publish") == 4
    pending = False
    for kind in kinds:
        assert not (pending and kind == "publish"), kinds
        pending = kind == "wait" or (pending and kind != "meet")
    assert not pending, kinds
