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


def test_lengths_are_read_ahead_only_behind_a_kernel_of_the_same_call():
    """Kernels that work out their piece from the lengths before they wait: one of the same call is in front, which has read them, or they wait."""
    text = (CSRC / "kv_weights.cu").read_text()
    kernels = text.split("__global__")[1:]
    ahead = [k for k in kernels if 0 <= k.find("find_piece(") < k.index('asm volatile("griddepcontrol.wait;"')]
    alone = [k for k in kernels if "kv_weights_sum_kernel(" in k.split("{")[0]]  # which a call without rows launches by itself
    assert len(kernels) == 3 and len(alone) == 1
    for k in ahead:
        assert "kv_weights_kept_kernel(" in k.split("{")[0]
    assert 0 < alone[0].index('if (p.tokens == 0) asm volatile("griddepcontrol.wait;"') < alone[0].index("find_piece(")
    launches = text[text.index("lce_status launch(const WeightsParams"):]
    # kept scores are only there where there were rows
    assert "p.tokens > 0 && bytes <= kMostScores" in text and launches.index("if (p.tokens > 0)") < launches.index("kv_weights_kept_kernel<")
