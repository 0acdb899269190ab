"""Orderings that a run cannot show to be there: checked in the text of the kernels."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_07609_b200", "csrc")


def _text(name):
    return open(os.path.join(CSRC, name)).read()


def _body(text, name):
    start = re.search(r"\b%s\([^;{]*\{" % name, text).end()
    depth, i = 1, start
    while depth:
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        i += 1
    return text[start:i]


def test_a_token_operand_made_by_a_pair_is_handed_over_at_cluster_scope():
    """CTA 1 writes its half with ordinary stores, CTA 0 issues the MMAs that read it: a release and an acquire whose scope
    holds both CTAs have to lie between (an arrival without a scope releases to its own CTA only)."""
    dec, tc = _text("gemm_dec.cuh"), _text("gemm_tc.cuh")
    arrive = re.search(r"if constexpr \(PAIR\) (\w+)\(&g_dec\.b_made\)", dec).group(1)
    wait = re.search(r"PAIR \? (\w+)\(c, &g_dec\.b_made", dec)
    assert wait, "pairs wait for the made operand with a wait of their own"
    out, back = _body(tc, arrive), _body(tc, wait.group(1))
    assert re.search(r"arrive\.release\.cluster|fence\.(release\.sync_restrict::shared::cta|acq_rel)\.cluster.*arrive\.relaxed\.cluster", out, re.S), arrive
    assert re.search(r"try_wait\.parity\.acquire\.cluster|try_wait\.parity\.relaxed\.cluster.*fence\.(acquire\.sync_restrict::shared::cluster|acq_rel)\.cluster",
                     back, re.S), wait.group(1)


def test_the_control_cta_leaves_by_one_threads_clock():
    """Threads that each compare their own clock leave the idle loop in different turns, and the CTA's barriers no longer match."""
    body = _body(_text("control.cuh"), "control_phase")
    by_thread_0 = "".join(re.findall(r"if \(tid == 0\) \{.*?\n    \}", body, re.S))
    assert body.count("- idle_t0") == by_thread_0.count("- idle_t0") == 1


def test_scheduler_and_phases_go_by_one_row_limit_for_small_steps():
    """The scheduler decides who applies RoPE, the phases who clears its input: two limits would drop one or the other."""
    control, dec = _text("control.cuh"), _text("gemm_dec.cuh")
    assert re.search(r"const int fuse = c\.dec_small && T <= DEC_SMALL_ROWS\b", control)
    assert re.search(r"bool dec_small\(.*\{ return c\.dec_small && T <= DEC_SMALL_ROWS; \}", dec)


def test_registers_of_a_tensor_memory_load_are_not_touched_before_the_wait():
    """They hold nothing until tcgen05.wait::ld.  So the wait is part of the load's statement, or it names the registers (+r) and stands
    behind the load in the same block: no branch, no way around a loop and no change of type between the two, each of which
    may be a copy."""
    texts = {f: re.sub(r"//[^\n]*", "", _text(f)) for f in sorted(os.listdir(CSRC)) if f.endswith((".cuh", ".cu"))}
    wrappers, n_loads = [], 0
    for text in texts.values():
        for st in re.finditer(r"asm volatile\((.*?)\);", text, re.S):
            code = st.group(1)
            if "tcgen05.ld." in code:
                n_loads += 1
                if "tcgen05.wait::ld" in code:
                    assert code.index("tcgen05.ld.") < code.index("tcgen05.wait::ld")
                    continue
                name, args = re.findall(r"void (\w+)\(([^{;]*)\) \{\s", text[:st.start()])[-1]
                assert re.search(r"uint32_t \(&\w+\)\[\d+\]", args), f"{name}: destinations of another type than the instruction's"
                wrappers.append(name)
            elif "tcgen05.wait::ld" in code:
                assert "+r" in code or "BLINK_RW" in code, "a wait that names no registers orders nothing that uses them"
    assert n_loads >= 2
    for name in wrappers:
        for f, text in texts.items():
            for call in re.finditer(r"\b%s\(([^;{]*), (\w+)\);" % name, text):
                depth, i = 0, call.end()
                while depth >= 0:   # to the end of the block that the load stands in
                    depth += {"{": 1, "}": -1}.get(text[i], 0)
                    i += 1
                head = text[:call.start()].rstrip()
                assert head[-1] in ";{}", f"{f}: {call.group(0)} under a condition"
                assert re.search(r"tmem_wait_ld\w*\([^;]*\b%s\b[^;]*\);" % call.group(2), text[call.end():i]), f"{f}: {call.group(0)} is not waited for in its block"


def test_copies_into_one_place_do_not_overtake_one_another():
    """Asynchronous copies of different groups have no order among themselves: before another is begun into the place of a warp's
    tile of draft probabilities, what was on its way there has landed."""
    body = _body(re.sub(r"//[^\n]*", "", _text("ops_verify.cu")), "blink_verify_draw_kernel")
    fetch = body[body.index("auto fetch_q = "):]
    fetch = fetch[:fetch.index("cp.async.commit_group")]
    assert 0 < fetch.find("cp.async.wait_group 0") < fetch.index("cp.async.c")
    assert body.count("cp.async.c") == fetch.count("cp.async.c") + 1      # (and its commit) nobody else copies there


def test_a_unit_is_written_over_when_all_warps_have_read_it():
    """The records of a CTA's units are used in turn.  Every warp says that it has read one, and whoever writes waits for all of them."""
    text = re.sub(r"//[^\n]*", "", _text("ops_attn_tiles.cu"))
    assert re.search(r"til_init\(&sh\.unit_empty\[i\], TIL_WARPS\)", text)
    read = text[text.index("auto unit_of = "):]
    read = read[:read.index("return t;")]
    at = [read.index(x) for x in ("wait(&sh.unit_full[slot]", "t = s_unit[slot]", "__syncwarp()", "til_arrive(&sh.unit_empty[slot])")]
    assert at == sorted(at)
    write = text[text.index("auto hand_out = "):]
    at = [write.index(x) for x in ("if (i >= TIL_UNITS) wait(&sh.unit_empty[i % TIL_UNITS], (uint32_t)(i / TIL_UNITS - 1) & 1u)", "s_unit[i % TIL_UNITS] = t",
                                   "til_arrive(&sh.unit_full[i % TIL_UNITS])")]
    assert at == sorted(at)
    assert text.count("s_unit[") == 2         # nobody else reads or writes them


def test_attention_that_gave_up_leaves_no_rows_that_look_like_results():
    """A call without a workspace of the caller's has no status that could be read: what a wait that ran out leaves undone has to show in the
    rows.  The first CTA that gives up fills all of them; none stores what a warp that gave up may have spoilt."""
    text = re.sub(r"//[^\n]*", "", _text("ops_attn_tiles.cu"))
    kernel = _body(text, "blink_attn_tiles_kernel")
    end = kernel[kernel.rindex("__syncthreads();"):]
    assert re.search(r"if \(sh\.dead\) til_give_up\(a, &sh\.first\);", end)
    assert re.search(r"const bool store = mine && ok && \*\(volatile int\*\)&sh\.dead == 0;", kernel) and kernel.count("store &&") + kernel.count("(store)") == 2
    assert "*(volatile int*)dead = 1" in text and text.count("BLINK_ETIMEDOUT") == 1     # the status is set by whoever fills the rows
    fill = _body(text, "til_give_up")
    assert "atomicExch(reinterpret_cast<int*>(a.ws), BLINK_ETIMEDOUT) == BLINK_OK" in fill and "0x7fff7fffu" in fill and "q.rows <= a.few" in fill


def test_operators_ask_the_device_for_its_sms():
    for f in sorted(os.listdir(CSRC)):
        if f.startswith("ops"):
            assert not re.search(r"\b148\b", re.sub(r"//[^\n]*", "", _text(f))), f


def test_operators_kernels_touch_nothing_before_their_own_wait():
    """A kernel may begin while those before it in the stream still run: what they wrote (the caller's lengths and queries, or an earlier kernel of
    the call) is sure to be seen behind its own griddepcontrol.wait only."""
    memory = re.compile(r"\ba\.(row_start|kv_len|table|temperature|u_pick|u_accept|draft|choice|chunks_of|logits|positions|slot_map|qkv|ctx_len|new_len|held|"
                        r"free_count|free_blocks|block_table|ws|q|out|pool)\b|\battn_req\(|\bws\[")
    found = 0
    for f in sorted(os.listdir(CSRC)):
        if not (f.startswith("ops_") and f.endswith(".cu")):
            continue
        text = re.sub(r"//[^\n]*", "", _text(f)).replace("int* status = reinterpret_cast<int*>(a.ws);", "")   # (its address)
        for name in re.findall(r"__global__ void (?:__launch_bounds__\([^)]*\) )?(\w+)\(", text) + (["ver_choose"] if f == "ops_verify.cu" else []):
            body = _body(text, name)
            waits = [m.start() for m in re.finditer(r"\bops_wait\(\);|\bops_begin\(\);|\bver_choose<", body)]
            touched = memory.search(re.sub(r"a\.pool\.(rep|hd|Hq|Hkv|n_blocks|dtype)\b", "shape", body[:waits[0]]))
            assert touched is None, (f, name, touched.group(0))
            found += 1
    assert found >= 11
