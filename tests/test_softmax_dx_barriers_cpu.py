"""The barriers in the walk of bf16 dx of long sums, as the compiler leaves them (no device)."""
import test_softmax_barriers_cpu as others


def test_every_barrier_of_the_walk_waits_for_the_reads_before_it(tmp_path):
    others.test_every_barrier_of_a_walk_waits_for_the_reads_before_it(tmp_path, 0, 2, 1)
