"""The profile summaries take the kernels of this library, and none whose name only holds one of theirs."""
import sqlite3

import rocprof_summary

KERNELS = ["void (anonymous namespace)::k_rows<1, 0, 8, false, false>((anonymous namespace)::RowArgs)",
           "void (anonymous namespace)::k_clip<0, 1, (anonymous namespace)::TensorBatch<11, true> >(float*)", "k_merge_sweep(int)",
           "(anonymous namespace)::k_sort_move((anonymous namespace)::SortArgs, (anonymous namespace)::Clearing)"]
OTHERS = ["void rocprim::ROCPRIM_400001_NS::detail::block_sort_kernel<256u, long>(long*)",
          "void rocprim::detail::trampoline_kernel<rocprim::detail::k_rows<int>, ns::k_sort_move>(int*)", "void at::native::radix_mask_join(int)"]


def test_only_the_librarys_kernels_are_summed_up(tmp_path):
    db = sqlite3.connect(tmp_path / "x_results.db")
    db.execute("create table kernels (name text, start integer, end integer)")
    db.execute("create table counters_collection (kernel_name text, counter_name text, value real, duration real)")
    for i, name in enumerate(KERNELS + OTHERS):
        db.execute("insert into kernels values (?, ?, ?)", (name, 1000 * i, 1000 * i + 500))
        db.execute("insert into counters_collection values (?, 'FETCH_SIZE', 2048, 1000)", (name,))
    db.commit()
    db.close()
    short = {"k_rows<1,0,8,false,false>", "k_clip<0,1,TensorBatch<11,tr", "k_merge_sweep", "k_sort_move"}
    for text in (rocprof_summary.trace(tmp_path / "x_results.db"), rocprof_summary.pmc([tmp_path / "x_results.db"])):
        assert {line.split()[0] for line in text.splitlines()[1:]} == short
    assert len(rocprof_summary.trace(tmp_path / "x_results.db", everything=True).splitlines()) == 1 + len(KERNELS + OTHERS)
