"""Rules of the kernels that no run shows: they concern launches whose bounded waits have given up, or a later change of a launch."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_17560_b200", "csrc")


def source(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


def test_a_pair_that_gave_up_orders_its_arrivals():
    """The pair GEMMs' last cluster barrier orders no memory, which is sound only while every arrival sent to the leader is one it
    waits for.  All four epilogues fence where they give a wait up, and the barrier acquires."""
    kernel = source("a3_gemm_persistent.cu").split("pair_t_kernel(", 1)[1].split("bool swiglu_pair_usable", 1)[0]
    assert re.search(r"give_up = \[\] \{ asm volatile\(\"fence.acq_rel.cluster;\"", kernel)
    left = re.findall(r"if \(!ep_ok\[0\]\) \{\s*(.*?)\s*\}", kernel, flags=re.S)
    assert len(left) == 4 == len(re.findall(r"ep_ok\[0\] = mbar_wait", kernel))
    assert all(re.match(r"give_up\(\);\s*(break|return false);", body) for body in left)
    barrier = source("a3_tc.cuh").split("cluster_sync_relaxed()", 1)[1].split("}", 1)[0]
    assert "arrive.relaxed" in barrier and "wait.acquire" in barrier


def test_launches_that_others_run_beside_are_ordinary():
    """rerotate_kernel and clear_ticket_kernel let their successors start early, which write before they wait: sound only because these
    two waited for everything before them.  Only rerotate itself says whether there is such a launch to run beside."""
    for name, kernel in (("a3_stream_kernels.cu", "rerotate_kernel"), ("a3_first_token.cu", "clear_ticket_kernel")):
        text = source(name)
        assert re.search(kernel + r"(<\w+, \w+>)?<<<", text)
        assert not re.search(r"launch_pdl(_cluster)?\([^;]*" + kernel, text)
    ticket = source("a3_first_token.cu").split("clear_ticket_kernel<<<")[1]
    assert ticket.split("launch_pdl(")[0].count(";") == 2  # the launch and its check, nothing queued in between
    for call in re.findall(r"enter_rows\([^;]*;", source("a3_api.cu")):
        last = call.rsplit(",", 1)[1].strip(" \n);")
        assert last in ("st", "recovering", "i == 0 && recovering"), last


def test_lengths_that_change_under_the_call_lead_nowhere():
    """paged_attention_kernel reads each length several times, and promises bounds even where another stream writes them meanwhile.  A warp's walk over its
    tiles, with the lengths of the scan and others read later; a rule that the source lacks is left out here too."""
    import itertools
    import random

    text = source("a3_paged_attention.cu")
    next_there = bool(re.search(r"if \(NT == 1 && cs \+ 1 < a\.n_seqs && count - i >", text))
    clamped = bool(re.search(r"xt = \(int\)min\(w0 - first0, \(unsigned\)cap / KT\)", text))

    def walk(scan, later, first_seq, skip, KT, cap):
        """Sequences whose queries are read, and the keys that tiles begin with."""
        tiles = lambda n: -(-n // KT)  # noqa: E731
        n_seqs, queries, keys = len(scan), [first_seq], []
        count = sum(tiles(x) for x in scan[first_seq:]) - skip
        xs, xn, xt = first_seq, scan[first_seq], min(skip, cap // KT) if clamped else skip
        q_seq, fresh = first_seq, True
        for i in range(count):
            cs, cn, ct = xs, xn, xt
            keys.append(ct * KT)
            if fresh:
                fresh = False
                if q_seq != cs:
                    q_seq = cs
                    queries.append(q_seq)
                if count - i > tiles(cn) - ct and (cs + 1 < n_seqs or not next_there):
                    q_seq += 1
                    queries.append(q_seq)
            fresh |= ct == tiles(cn) - 1
            xt += 1
            if xt * KT >= xn:
                xt = 0
                while True:
                    if xs == n_seqs - 1:
                        xn = 0
                        break
                    xs += 1
                    xn = later[xs]
                    if xn > 0:
                        break
        return queries, keys

    rng = random.Random(0)
    for scan, later in itertools.product(itertools.product((0, 1, 16, 33, 64), repeat=3), repeat=2):
        if scan[0]:
            queries, keys = walk(scan, later, 0, 0, 16, 64)
            assert all(0 <= q < 3 for q in queries) and all(k <= 64 + 16 for k in keys), (scan, later, queries)
    for _ in range(500):
        cap = rng.choice((64, 2 ** 31 - 2 ** 16))
        scan, later = [[rng.choice((0, 1, 16, 500)) % (cap + 1) for _ in range(6)] for _ in range(2)]
        # a stretch whose first sequence and first tile were written by two threads that saw different lengths
        queries, keys = walk(scan, later, rng.randrange(6), rng.choice((0, 1, 3, 2 ** 28)), 16, cap)
        assert all(0 <= q < 6 for q in queries) and all(k <= cap + 16 for k in keys)
    # the first tile of a stretch far along a line of 2^34 slots: its first key has to fit 32 bits
    assert clamped


def test_lanes_meet_before_a_barrier_of_a_cluster():
    """The aligned forms of the cluster barrier want a warp's lanes together, and both kernels reach it from loops that lanes leave at different times."""
    for name in ("a3_paged_attention.cu", "a3_logprobs.cu"):
        text = source(name)
        barriers = [m.start() for m in re.finditer(r"asm volatile\(\"barrier\.cluster\.(arrive|wait)", text)]
        assert barriers and all(re.search(r"__syncwarp\(\);\s*$", text[:at]) for at in barriers), name


def test_decoding_reads_nothing_as_read_only_that_the_launch_before_may_write():
    """These kernels begin while the launch before them may still run.  A read-only load says that nobody writes during the kernel, and may be moved in front
    of the wait: it is for the table of angles, which is written when a handle is made."""
    for name in ("a3_paged_append.cu", "a3_paged_attention.cu", "a3_logprobs.cu"):
        loads = re.findall(r"(?:__ldg|ld\.global\.nc)\S*", source(name))
        assert all(x.startswith("__ldg(tr") for x in loads), (name, loads)
