"""The build counts, in the device assembly, the reads from memory that a wait further on counts on.  The scanner against hand-written
fragments."""
from paper_2311_15269_amd.build import miscounted_reads

BEGIN, END, WAIT = "\t; counted reads begin\n", "\t; counted reads end %d\n", "\ts_waitcnt vmcnt(%d) ; counted\n"
READ, COPY = "\tglobal_load_dwordx4 v[0:3], v4, s[0:1]\n", "\tglobal_load_lds_dwordx4 v[0:1], off\n"
OVER = ".Lfunc_end0:\n"


def test_stretches_that_hold_what_they_promise_pass():
    assert miscounted_reads(BEGIN + READ + "\tv_add_u32 v4, v4, v5\n" + READ + END % 2 + BEGIN + COPY * 4 + END % 4 + WAIT % 6 + OVER) == []
    assert miscounted_reads(READ + "\ts_waitcnt vmcnt(0)\n" + OVER) == []


def test_too_few_reads_are_reported():
    assert miscounted_reads(BEGIN + READ + END % 2 + WAIT % 2 + OVER) == ["3: 1 reads since line 1, not 2"]
    assert len(miscounted_reads(BEGIN + END % 4 + COPY * 4 + OVER)) == 1          # (moved behind the end)
    assert miscounted_reads(BEGIN + READ + "\t; global_load_dword\n" + "\tds_read_b128 v[0:3], v4\n" + END % 2 + OVER) != []


def test_a_stretch_in_pieces_is_reported():
    assert miscounted_reads(BEGIN + READ + "\ts_cbranch_vccnz .LBB0_2\n" + READ + END % 2 + OVER) != []
    assert miscounted_reads(BEGIN + READ + ".LBB0_2:\n" + READ + END % 2 + OVER) != []
    assert miscounted_reads(BEGIN + READ + BEGIN + READ + END % 1 + OVER) != []
    assert miscounted_reads(BEGIN + READ + OVER) != [] and miscounted_reads(READ + END % 1 + OVER) != []


def test_a_counted_wait_without_marked_reads_is_reported():
    assert miscounted_reads(COPY + READ + WAIT % 1 + OVER) == ["3: a counted wait, but no reads are marked"]
    assert miscounted_reads(BEGIN + READ + END % 1 + WAIT % 1 + OVER + READ + WAIT % 1 + OVER) != []
