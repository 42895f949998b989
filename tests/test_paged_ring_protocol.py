"""The ring of operands that the two producers and the two MMA issuers of the chunk kernel share (bf16 pages, csrc/paged_chunk.cuh), walked through
on the CPU.  A wait by parity also passes for a barrier that is two rounds behind; the kernel relies on that never happening, which holds as long as
every issuer releases operands in their order.  Letting it happen on a GPU is not an option for a test (a copy would land in a slot that is in use), so all
interleavings of a few segments are gone through here, and the rule is held against the kernel's source."""
import itertools
import os
import re

import pytest

from paper_2510_07651_b200 import build

NS = 3                                           # slots of the ring


def _numbers(segments):
    """The operands in the order in which issuers take them: (kind, warpgroups that see it), and the numbers of every producer's, as the kernel counts them."""
    ops, k_ops, v_ops, base = {}, [], [], 0
    for n, cnt0, cnt1 in segments:
        for i in range(n):
            k = 2 * base + (2 * i - 1 if i > 0 else 2 * i)
            v = 2 * base + (2 * i + 2 if i + 1 < n else 2 * i + 1)
            sees = (i < cnt0, i < cnt1)
            assert k not in ops and v not in ops
            ops[k], ops[v] = ("K", sees), ("V", sees)
            k_ops.append(k)
            v_ops.append(v)
        base += n
    assert sorted(ops) == list(range(2 * base))
    return [ops[j] for j in range(2 * base)], k_ops, v_ops


def walk(segments, in_order):
    """Goes through every state that two producers, two issuers, their MMAs and two softmax warpgroups can reach.  in_order: an issuer releases what it does
    not see by a commit, behind its MMAs; else at once.  Returns (a producer's wait passed for an earlier round, a state without a way on)."""
    ops, *producers = _numbers(segments)
    n = len(ops)
    seen_before = [[[0] * (n + 1) for _ in "KV"] for _ in range(2)]       # [w][kind][j]: operands of a kind below j that warpgroup w sees
    for w in range(2):
        for x, kind in enumerate("KV"):
            for j in range(n):
                seen_before[w][x][j + 1] = seen_before[w][x][j] + (ops[j][0] == kind and ops[j][1][w])
    early = stuck = False

    def released(j, w, issued, done):
        """Has issuer w released operand j?  issued, done: operands that it has gone through, and of which the MMAs (and commits) are complete."""
        return j < done or (not in_order and j < issued and not ops[j][1][w])

    # producers' positions; per issuer: operands gone through, complete; per softmax warpgroup: S read, P written
    start = (0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    todo, known = [start], {start}
    while todo:
        state = todo.pop()
        at, issued, done, read, wrote = state[0:2], state[2:4], state[4:6], state[6:8], state[8:10]
        ways = []
        for p in range(2):
            if at[p] < len(producers[p]):
                k = producers[p][at[p]]
                turns = sum(released(j, w, issued[w], done[w]) for j in range(k % NS, n, NS) for w in range(2)) // 2
                if turns % 2 == (k // NS) % 2:                        # what the wait can see
                    if turns == k // NS:
                        ways.append(state[:p] + (at[p] + 1,) + state[p + 1:])
                    else:
                        early = True
        for w in range(2):
            j = issued[w]
            if j < n:
                kind, sees = ops[j][0], ops[j][1][w]
                p = "KV".index(kind)
                full = j in producers[p][:at[p]]
                s, v = seen_before[w][0][j], seen_before[w][1][j]
                ready = full and (not sees or (read[w] >= s if kind == "K" else wrote[w] > v))       # S is free; P is there
                if ready:
                    ways.append(state[:2 + w] + (j + 1,) + state[3 + w:])
            if done[w] < issued[w]:
                ways.append(state[:4 + w] + (done[w] + 1,) + state[5 + w:])
            if seen_before[w][0][done[w]] > read[w] and read[w] == wrote[w]:             # the next S is complete
                ways.append(state[:6 + w] + (read[w] + 1,) + state[7 + w:])
            if read[w] > wrote[w] and seen_before[w][1][done[w]] >= wrote[w]:            # P V of the tile before is complete
                ways.append(state[:8 + w] + (wrote[w] + 1,) + state[9 + w:])
        if not ways and not (issued == done == (n, n)):
            stuck = True
        for s in ways:
            if s not in known:
                known.add(s)
                todo.append(s)
    return early, stuck


def _segments(longest):
    """What a segment of 1 to `longest` tiles may look like: warpgroup 1 sees all of them or, behind a full row tile's last rows, none; warpgroup 0 sees
    all or (causal) one fewer, or only the first ones of a segment that begins late in a list."""
    for n in range(1, longest + 1):
        yield from dict.fromkeys([(n, n, n), (n, n, 0), (n, n - 1, n), (n, max(n - 2, 0), n)])


@pytest.mark.parametrize("pair", list(itertools.product(_segments(3), repeat=2)) + [((4, 4, 4), (4, 4, 0)), ((4, 4, 0), (4, 3, 4)), ((1, 1, 0), (5, 5, 0)), ((5, 5, 0),), ((5, 4, 5),)])
def test_no_wait_passes_for_an_earlier_round(pair):
    assert walk(pair, in_order=True) == (False, False)


@pytest.mark.parametrize("pair", [((4, 4, 4), (4, 4, 0)), ((2, 1, 2), (3, 3, 3))])
def test_the_walk_finds_releases_out_of_order(pair):
    """With plain arrivals for what a warpgroup does not see, the slot of the operand before may still be in use two rounds on."""
    early, _ = walk(pair, in_order=False)
    assert early


def test_issuers_release_by_commits_alone():
    text = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, "paged_chunk.cuh")).read())
    issuers = text[text.index("const bool leader = elect_one();"):text.index("} else if (warp < 12)")]
    assert issuers.count("tc_commit(bar(L::EMPTY + slot))") == 4 and "mbar_arrive" not in issuers


def test_nothing_is_under_way_when_a_cta_leaves():
    """The last operand of every slot has landed and has been released by both issuers, whose commits arrive on barriers in the CTA's shared memory."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, "paged_chunk.cuh")).read())
    drain = re.search(r"if \(j \+ n >= NS && recent\[j\] \+ NS >= 2 \* n\) \{(.*?)\n\s*\}", text, re.S)[1]
    assert "mbar_wait(bar(L::FULL + recent[j] % NS), (recent[j] / NS) & 1u)" in drain and "all_wait(L::EMPTY + recent[j] % NS, recent[j] / NS, __LINE__)" in drain
    assert re.search(r"for \(uint32_t k = n > NS \? n - NS : 0u; k < n && !fail_site; \+\+k\) \(void\)all_wait\(L::EMPTY \+ k % NS, k / NS, __LINE__\)", text)
