"""Which keys count, and the rows' terms, are ordinary stores of one warp that others read:
each reader has to wait at that warp's own barrier.  A commit of the tensor cores that came
later in another thread does not stand for it.  Read from the sources, since a run on a GPU
shows a missing order only by chance."""
import os

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_22922_gb300", "csrc")

# source, what begins the readers' loop over tiles, what they read, the writer's barrier
READERS = [("attend_short.cu", "const int group = warp >> 2", "bars.most[", "bars.fixed["),
           ("attend_tc.cu", "} else if (warp < kSoftWarps", "bars.mask[", "bars.mask_ready["),
           ("attend_grad_short.cu", "const int group = warp >> 2", "bars.bias[", "bars.kv_fixed["),
           ("attend_grad_tc.cu", "const int quad = warp & 3, half = warp >> 2;", "bars.lse2[", "bars.fixed["),
           ("attend_grad_tc.cu", "const int quad = warp & 3, half = warp >> 2, r =", "bars.mask[", "bars.fixed[")]


def test_readers_wait_for_the_writer():
    for name, begin, read, barrier in READERS:
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        assert text.count(begin) == 1, (name, begin)
        at = text.index(begin)
        first = text.index(read, at)
        wait = text.find("w.wait(smem_addr(&" + barrier, at, first)
        assert wait > 0, "%s reads %s] before it waits for %s]" % (name, read, barrier)
