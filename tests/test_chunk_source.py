"""Rules that the chunk attention kernel keeps, read in its source (no GPU)."""
import pathlib
import re

import paper_2607_20507_gb300 as package

SOURCE = pathlib.Path(package.__file__).parent / "csrc" / "chunk_attention.cu"

ALIGNED = re.compile(r"\btmem_(ld32|ld16|st16|ld_done|st_done)\b|tcgen05\.(alloc|dealloc)")
# what may leave the threads of a warp apart: a branch by lane or by row, and barriers of several warps (which bring
# threads together, but not so that an aligned instruction may follow)
PARTS = re.compile(r"if \(lane|if \(!?token|if \(threadIdx|\b(pair_sync|pair_any|all_sync|hide|mbar_wait_bounded)\(|__syncthreads\(\)|__shfl")
TOGETHER = re.compile(r"__syncwarp\(\)|\bwait\(&bars")


def kernel():
    text = SOURCE.read_text()
    body = text[text.index("chunk_attention_kernel(const"):text.index("// ---", text.index("tcgen05.dealloc"))]
    return [re.sub(r"//.*", "", line) for line in body.split("\n")]


def test_warps_are_together_at_instructions_of_whole_warps():
    """tcgen05.ld, st, wait, alloc and dealloc are .sync.aligned: all threads of the warp execute the same one.  In the
    order of the source, nothing that may leave a warp's threads apart stands between them and the last __syncwarp (wait()
    ends with one)."""
    apart, seen = False, 0
    for line in kernel():
        if TOGETHER.search(line):
            apart = False
        if ALIGNED.search(line):
            seen += 1
            assert not apart, line.strip()
        if PARTS.search(line):
            apart = True
    assert seen >= 12


def test_no_thread_leaves_a_round_that_ends_with_such_an_instruction():
    """Inside the loops over a piece's dims a thread without a row passes over its stores; it does not go on by itself."""
    text = "\n".join(kernel())
    assert not re.search(r"if \((token|lane)[^\n]*\)\s*(continue|break);", text)
    end = text[text.index("for (int again = 0;;"):]
    loop = end[end.index("for (int q = 0; q < 2; ++q)"):]
    assert re.match(r"[^;]*;[^;]*;[^;]*;\s*__syncwarp\(\);\s*tmem_ld16", loop)


def test_wide_stores_go_where_32_byte_alignment_is_known():
    """Stores of 32 bytes: to the workspace, which is aligned to 256, and to an output in the kernel for such outputs, which
    the host takes by the address.  An output is promised 16."""
    text = SOURCE.read_text()
    assert len(re.findall(r"\.global\.v8\.", text)) == 1 and "void store32(float* p" in text
    assert re.findall(r"\bstore32\((?!float\* p)([^,]+),", text) == [
        "reinterpret_cast<float*>(p)", "p.part_o + at_row * kD + part * 32 + q * 16 + j * 8"]
    assert re.search(r"if constexpr \(kWide\) \{\s*store32\(reinterpret_cast<float\*>\(p\)", text)
    assert "wide_out = reinterpret_cast<uintptr_t>(out) % 32 == 0" in text
    assert len(re.findall(r"\bstore_out<kWide>\(", text)) == 3


def test_the_place_of_a_count_is_one_of_the_grid():
    """Cuts::first() names the word in which a block's finished tiles are counted.  Where starts decrease, rows count several
    times and the weights may pass their type, so its quotient may be anything: it is bounded before it becomes an int (a
    quotient of 2^31 or more by a small share would be a negative one)."""
    text = SOURCE.read_text()
    first = text[text.index("int first() const {"):]
    first = first[:first.index("\n    }\n")]
    assert re.search(r"const W at = .*quotient\(.*quotient\(", first) and not re.search(r"\(int\)\s*quotient", first)
    assert "int c = at < (W)ctas ? (int)at : ctas - 1;" in first and "return c;" in first
    # a model of it: any place of the weight, any share, 32 bits
    mask = (1 << 32) - 1
    for each in (0, 1, 2, 7, 1 << 20, mask):
        for over in (0, 1, 151):
            for x0 in (0, 1, 150, 1 << 31, mask - 1, mask):
                more = (each + 1) * over & mask
                if x0 < more:
                    at = x0 // ((each + 1) & mask) if (each + 1) & mask else mask
                else:
                    at = over + ((x0 - more) // each if each else mask) & mask
                c = at if at < 152 else 151
                assert 0 <= c < 152


def test_every_wait_is_bounded_and_every_role_comes_to_the_end():
    """Waits on mbarriers: wait() and wait_lane(), which go on to the bounded one that the self-test lets run out and raise the
    block's flag, and that one itself.  No thread leaves the kernel early, so that all meet the last barrier, with the products
    of either issuing warp and the copies of the producers complete, before tensor memory is given back."""
    text = SOURCE.read_text()
    body = "\n".join(kernel())
    assert not re.search(r"mbar_(try|test)_wait|mbarrier\.(try|test)_wait", body)
    for name in ("wait_lane", "wait"):
        f = text[text.index(f"void {name}(uint64_t* bar"):]
        assert "if (!mbar_try_wait(bar, parity) && !*dead && !mbar_wait_bounded(bar, parity))" in f[:f.index("\n}\n")]
    assert "!mbar_wait_bounded(" in (SOURCE.parent / "selftest.cu").read_text()
    look = body[body.index("auto look = [&](int b) {"):]      # (a function of its own)
    assert body.count("return;") == look[:look.index("};")].count("return;") == 1 and "exit;" not in body
    end = body[body.rindex("__syncthreads()"):]
    assert "tcgen05.dealloc" in end and body.index("mbar_wait_bounded(&bars.drained, 0)") < body.rindex("__syncthreads()")
    roles = body[body.index("if (warp == kKvWarp) {"):]
    producers = roles[:roles.index("const int m = warp == kMmaWarp")]
    assert producers.count("if (!alive(&s_dead)) break;") == 2     # nothing more into places that may be in use
    assert "mbar_wait_bounded(&bars.kv_full" in producers and "mbar_wait_bounded(&bars.q_full" in producers
