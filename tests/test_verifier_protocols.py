"""What the verifier's kernels rely on between warps and thread blocks, checked on the CPU against their source: faults of this kind show
themselves by chance or not at all when they run."""
import os
import random
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_20375_b200", "csrc")


def _kernel(source, name):
    """The text of a kernel without comments, from its name to the closing brace in the first column."""
    with open(os.path.join(CSRC, source)) as f:
        text = f.read()
    text = text[re.search(r"__global__[^;{]*\b" + name + r"\(", text).start():]
    return re.sub(r"//[^\n]*", "", text[:text.index("\n}\n")])


def test_the_walk_writes_to_other_blocks_once_they_have_begun():
    """Shared memory of another block of the cluster may be written when that block is known to run: every thread arrives at the cluster's
    barrier and waits for all before its first exchange.  The arrival comes before anything that takes time, so that the wait is short."""
    k = _kernel("verify.cu", "verify_kernel")
    first = re.search(r"\bexchange\((?!uint64_t)", k).start()  # (behind the definition of the lambda)
    arrive, wait = (k.find(f"barrier.cluster.{x}") for x in ("arrive", "wait"))
    assert 0 <= arrive < k.index("pdl_wait()") < wait < first
    # neither stands in a branch: the braces around them are the kernel's own
    for at in (arrive, wait):
        assert k[:at].count("{") - k[:at].count("}") == 1 + k[:at].count("namespace {")


def _pieces_of_two_row_tiles(slots, pieces, rng):
    """Eight softmax warps (the first four a stream) along a CTA's pieces of two row tiles, each with a row of V that one warp of the first
    stream takes out.  Its flag is one of `slots`, piece by piece.  The first thing that goes wrong, or None."""
    at_q, met, flag, wrong = [0] * pieces, [0] * pieces, [0] * slots, []
    finder = [rng.randrange(4) for _ in range(pieces)]

    def warp(w):
        for n in range(pieces):
            at_q[n] += 1                     # its rows of Q are there
            yield lambda: True
            if w == finder[n]:               # V is looked through ahead of the first scores
                flag[n % slots] = n + 1
            yield lambda n=n: at_q[n] == 8   # the first scores: products begin when all eight have arrived
            met[n] += 1                      # (behind the weights of the tile the streams meet)
            yield lambda n=n: met[n] == 8
            yield lambda: True               # the end of the piece is reached at any time
            if flag[n % slots] != n + 1:
                wrong.append(f"warp {w} adds nothing in piece {n}")

    warps = {w: warp(w) for w in range(8)}
    waits = {w: next(warps[w]) for w in warps}
    while waits:
        ready = [w for w in waits if waits[w]()]
        if not ready:
            return "nobody can go on"
        w = rng.choice(ready)
        try:
            waits[w] = next(warps[w])
        except StopIteration:
            del waits[w]
    return wrong[0] if wrong else None


def test_rows_of_v_that_were_taken_out_are_known_to_all_warps_of_their_piece():
    """A warp that runs ahead may take out a row of the next piece's V while others have yet to look at this piece's flag."""
    k = _kernel("tree_attn.cu", "tree_attn_kernel")
    with open(os.path.join(CSRC, "tree_attn.cu")) as f:
        found = re.search(r"constexpr int kSpoiltPieces = (\d+);", f.read())
    slots = int(found.group(1)) if found else 1
    uses = re.findall(r"spoilt\[([^\n]*?)\]\s*==?\s", k)
    assert len(uses) == 3 and sum("n_piece % kSpoiltPieces" in u for u in uses) == 2, uses  # (and all are cleared in the beginning)
    rng = random.Random(1)
    assert any(_pieces_of_two_row_tiles(1, 6, rng) for _ in range(200))  # one flag is not enough
    for _ in range(2000):
        assert _pieces_of_two_row_tiles(slots, 6, rng) is None
