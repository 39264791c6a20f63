"""How the tensor-core kernel of kv_attend deals out its registers, read from its source: no GPU is needed, and a wrong split must
not run on one (a warpgroup that takes up more registers than the launch has left over waits for good)."""
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_26968_b200", "csrc", "kv_attend_tiles.cu")


def test_each_warpgroup_has_one_instruction():
    """All warps of a warpgroup have to execute the same setmaxnreg: one that gives registers up, one that takes them."""
    forms = re.findall(r"setmaxnreg\.(\w+)\.sync\.aligned\.u32 (\d+);", open(SOURCE).read())
    assert sorted(f for f, _ in forms) == ["dec", "inc"], forms


def test_shares_are_what_the_launch_has():
    text = open(SOURCE).read()
    forms = dict(re.findall(r"setmaxnreg\.(\w+)\.sync\.aligned\.u32 (\d+);", text))
    give, take = int(forms["dec"]), int(forms["inc"])
    # one warpgroup of copies and products, two of the softmax; 384 threads of at most 65,536 registers, in eights
    launch = 65_536 // 384 // 8 * 8
    assert give % 8 == 0 and take % 8 == 0 and give < launch < take
    assert 128 * (give + 2 * take) <= 384 * launch
    # the launch is refused where the compiler has used fewer
    assert text.count(">= 128 * (%d + 2 * %d)" % (give, take)) == 2
