"""The AdamW step over lists long enough for the kernels that take several blocks per warp, in full against the formula in 64 bits
(the bounds of test_gpu_adamw.py).  The threshold is read from the source, so that moving it cannot drop them."""
import os
import re

import pytest

import paper_1906_03707_b200 as hb
from paper_1906_03707_b200.build import CSRC, build as build_library
from test_gpu_adamw import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _few_blocks():
    """The most blocks of a launch that are still taken one at a time, as the source has it."""
    text = open(os.path.join(CSRC, "hag_adamw.cu")).read()
    value = lambda name: re.search(rf"constexpr int(?:64_t)? (?:\w+ = [^,;]+, )*{name} = ([^;,]+)[;,]", text).group(1)  # noqa: E731
    names = {"kSms": int(value("kSms")), "kAdamWarps": int(eval(value("kAdamThreads"))) // 32}
    return int(eval(value("kFewBlocks"), names))


FEW = _few_blocks()
# beyond the threshold by half: one long tensor that ends inside a block and inside a unit of several blocks, short ones between
LONG = 256 * (FEW + FEW // 4) + 3
LISTS = [[LONG, 70_001, 7, 257, 1_000_000, 0, 255], [70_001, 1, LONG // 2, 512, LONG // 2 + 300, 65_537, 31],
         [1, 300, 1025, 1024, 1023] * 12 + [LONG, 5 * 256, 6 * 256 + 1, 7 * 256 - 1, 4 * 256] * 2]


@pytest.fixture(scope="module", autouse=True)
def _library():
    build_library()
    hb.load_library()
    assert torch.cuda.is_available(), "the parity tests need a CUDA device"


def _blocks(lengths):
    return sum(-(-m // 256) for m in lengths)


@pytest.mark.parametrize("which", range(len(LISTS)))
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed", "odd"])
def test_long_lists(which, bits, kind):
    lengths = LISTS[which]
    assert _blocks(lengths[-64:]) > FEW                        # of one launch, whichever tensors it begins with
    Case(20 + which, lengths, (kind,), bits).check(step=3)
    case = Case(30 + which, lengths, (kind,), bits)
    copies = [None if t % 3 == 1 else torch.empty(m, dtype=BF16, device="cuda") for t, m in enumerate(lengths)]
    norm = hb.grad_norm(case.grads)
    case.check(norm=norm, max_norm=0.2 * float(norm), decay=[0.01 * (t % 3) for t in range(len(lengths))], copies=copies, eps=1e-4)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("offset,goffset", [(1, 1), (0, 3), (2, 0), (4, 4)])
def test_long_lists_off_the_vector_boundary(bits, offset, goffset):
    """Some types are off their vectors, others not, and with them one launch holds both forms."""
    lengths = [LONG // 2 + 129, 1025, LONG // 2 + 1, 3]
    assert _blocks(lengths) > FEW
    case = Case(40, lengths, ("mixed", "bf16", "f32", "odd"), bits, offset, goffset)
    norm = hb.grad_norm(case.grads)
    wide = torch.full((lengths[0] + 16,), 3.0, device="cuda", dtype=BF16)
    case.check(norm=norm, max_norm=0.7 * float(norm), copies=[wide[offset:offset + lengths[0]], None, None, None])
    assert (wide[:offset] == 3).all() and (wide[offset + lengths[0]:] == 3).all()


@pytest.mark.parametrize("bits", [8, 32])
def test_long_lists_with_missing_gradients(bits):
    case = Case(50, [5000, LONG, 300, 1_000_003, 77], ("f32", "bf16"), bits)
    case.check(missing=(0, 3))
    case.check(missing=(1,), step=8)
