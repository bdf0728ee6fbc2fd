"""CPU check of how the prefill kernel over a paged cache hands its items from the producer to the
other warps: every order in which producer, MMA issuer and the two softmax warpgroups may run, for a
CTA of 256 channels (one tile of rows; the warpgroups take tiles of slots in turn, so that an item of
one tile of slots needs no weights of the second). Whether the producer waits for the readers of the
record that it is about to write is read from the kernel's source."""
import itertools
import os
import re

import pytest

from paper_2606_07878_gb300 import still

SOURCE = os.path.join(os.path.dirname(still.LIB_PATH), "csrc", "paged_prefill.cu")
END = -1


def _awaits_readers():
    """(before an item's record is written, before the one that ends the items)"""
    src = open(SOURCE).read()
    init = re.findall(r"mbar_init\(&seen\[[01]\], 8\);", src)
    reads = re.search(r"const PfItem it = shown\[n_items & 1\];\s*__syncwarp\(\);\s*"
                      r"if \(lane == 0\) mbar_arrive\(&seen\[n_items & 1\]\);", src)
    wait = r"&seen\[n_items & 1\], \(\(n_items >> 1\) - 1\) & 1"
    item = re.search(wait + r".{,120}shown\[n_items & 1\] = it;", src, re.S)
    end = re.search(wait + r".{,240}shown\[n_items & 1\]\.k0 = shown\[n_items & 1\]\.k1 = 0;", src,
                    re.S)
    both = len(init) == 2 and bool(reads)
    return both and bool(item), both and bool(end)


def _programs(tiles, awaits):
    """Lists of steps: ("wait", barrier, parity), ("arrive", barrier), ("write", n, value) and
    ("read", n, value) of record n & 1."""
    producer, issuer, groups = [], [], ([], [])
    uses = [0, 0]  # of the buffers of S
    for n, k in enumerate(tiles + [0]):
        if n > 0:
            producer.append(("wait", "qfree", (n - 1) & 1))
        if n > 1 and awaits[k == 0]:
            producer.append(("wait", f"seen{n & 1}", ((n >> 1) - 1) & 1))
        producer += [("write", n, n if k else END), ("arrive", f"qfull{n & 1}")]
        issuer += [("wait", f"qfull{n & 1}", (n >> 1) & 1), ("read", n, n if k else END)]
        for g in groups:
            g += [("wait", f"qfull{n & 1}", (n >> 1) & 1), ("read", n, n if k else END),
                  ("arrive", f"seen{n & 1}")]
        if k == 0:
            break
        start = list(uses)

        def make_s(i):
            issuer.append(("arrive", f"sfull{i & 1}"))
            if i + 1 == k:
                issuer.append(("arrive", "qfree"))

        for i in range(min(2, k)):
            make_s(i)
        for i in range(k):
            b = i & 1
            issuer.append(("wait", f"pfull{b}", uses[b] & 1))
            if i == 0 and n > 0:
                issuer.append(("wait", "ofree", (n - 1) & 1))
            issuer.append(("arrive", f"pvdone{b}"))
            uses[b] += 1
            if i + 2 < k:
                make_s(i + 2)
        for w, g in enumerate(groups):
            used = list(start)  # of this warpgroup's buffer, of the other's
            for i in range(w, k, 2):
                g.append(("wait", f"sfull{w}", used[w] & 1))
                if i > 0:  # the running maximum
                    before = start[1 - w] + (i + 1) // 2
                    g.append(("wait", f"mb{1 - w}", (before - 1) & 1))
                g += [("arrive", f"mb{w}"), ("arrive", f"pfull{w}")]
                used[w] += 1
            last = (k - 1) & 1
            if last != w:
                g.append(("wait", f"mb{1 - w}", (uses[1 - w] - 1) & 1))
            g += [("wait", f"pvdone{last}", (uses[last] - 1) & 1), ("arrive", "lb"),
                  ("wait", "lb", n & 1), ("arrive", "ofree")]
    return [producer, issuer, *groups]


COUNTS = {"lb": 2, "ofree": 2, "seen0": 2, "seen1": 2}  # arrivals of a phase (a warpgroup is one)


def _fault(programs):
    """What some order of the steps comes to: None, or a record read that is another item's, or an
    order in which nobody can go on."""
    names = sorted({s[1] for p in programs for s in p if s[0] in ("wait", "arrive")})
    index = {name: i for i, name in enumerate(names)}
    first = ((0,) * len(programs), (0,) * len(names), (None, None))
    seen, todo = {first}, [first]
    while todo:
        at, arrived, record = todo.pop()
        moved = False
        for who, program in enumerate(programs):
            if at[who] == len(program):
                continue
            kind, what, value = (program[at[who]] + (None,))[:3]
            now, here = arrived, record
            if kind == "wait":
                phases = arrived[index[what]] // COUNTS.get(what, 1)
                if (phases & 1) == value:  # the phase of that parity is not complete
                    continue
            elif kind == "arrive":
                i = index[what]
                now = arrived[:i] + (arrived[i] + 1,) + arrived[i + 1:]
            elif kind == "write":
                here = (value, record[1]) if what % 2 == 0 else (record[0], value)
            elif record[what & 1] != value:
                return f"reader {who} of item {what} finds {record[what & 1]}"
            moved = True
            state = (at[:who] + (at[who] + 1,) + at[who + 1:], now, here)
            if state not in seen:
                seen.add(state)
                todo.append(state)
        if not moved and any(a < len(p) for a, p in zip(at, programs)):
            return f"nobody goes on at {at}"
    return None


@pytest.mark.parametrize("tiles", [list(x) for k in (1, 2, 3, 4)
                                   for x in itertools.product((1, 2, 3), repeat=k)])
def test_every_warp_reads_the_item_that_it_was_shown(tiles):
    assert _fault(_programs(tiles, _awaits_readers())) is None


def test_the_join_finds_a_record_of_every_cta():
    """A CTA that leaves early has said before that it splits no item: the join reads the workspace,
    which nobody cleared, by these records."""
    src = re.sub(r"//[^\n]*", "", open(SOURCE).read())
    kernel = src[src.index("paged_prefill_kernel("):src.index("paged_join_kernel(")]
    record = kernel.index("f.split[cta].last = f.split[cta].first = cta;")
    assert record < kernel.index("return;")


def test_the_search_finds_a_record_written_too_early():
    """Without the wait for its readers an item of one tile of slots is overtaken: the search sees
    what it looks for."""
    assert "finds" in _fault(_programs([1, 1, 1], (False, False)))
    assert _fault(_programs([1, 1, 1], (True, False))) is not None
