"""What a plan of kv16_plan says, checked as a whole: every page of every record and every large run is one worker's, and the
merge looks for partial results where those workers put them.  Worked out here from the lengths and the two numbers of
workers that the plan's header holds; works on a workspace's bytes, wherever they were made."""
import os
import re

import numpy as np

_text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_12707_gb300", "csrc", "kvd_kv16_plan.h")).read()
_consts = {n: int(v.rstrip("u"), 0) for n, v in re.findall(r"\b(k\w+) = (0x[0-9a-f]+u|\d+)\b", _text)}
P, WARPS, COLS, TILE = 16, _consts["kAttnWarps"], _consts["kRecordCols"], _consts["kTileRows"]
WIDE, NARROW = _consts["kWideCost"], _consts["kNarrowCost"]                      # cost of a page,
OPENS = {WIDE: _consts["kWideStart"], NARROW: _consts["kNarrowStart"]}           # and pages that opening a job counts
MADE, GAVE_UP = _consts["kPlanMagic"], _consts["kPlanGaveUp"]

_record = [(n, "<i4") for n in ("req", "len", "pages", "row0", "rows", "unit", "col", "pad")]
_run = [("req", "<i4"), ("len", "<i4"), ("pages", "<i4"), ("rows", "<i4"), ("cost", "<i8"), ("rows_before", "<i4"), ("chunks", "<i4")]
_segment = [(n, "<i4") for n in ("pages", "valid", "wide", "head", "row0", "rows", "rows0", "first")] + [("entry", "<i8")]
_shares = [("each", "<i8"), ("inverse", "<f4"), ("n", "<i4")]
HEADER = np.dtype([(n, "<i4") for n in ("magic", "batch", "hq", "hkv", "dim", "grid", "max_seqs", "max_pages", "prefix_ctas", "pad")]
                  + [("units", _shares), ("cost", _shares)])
RECORD, RUN = np.dtype(_record), np.dtype(_run)
ROW = np.dtype([("own", "<i8"), ("prefix", "<i8")] + [(n, "<i4") for n in ("own_count", "prefix_count", "step", "stream_step")])
WARP = np.dtype([(n, "<i4") for n in ("worker", "rec", "head", "page", "count")] + [("r", _record), ("pad", "<i4", 3)])
CTA = np.dtype([("run", "<i4"), ("job", "<i4"), ("end", "<i8"), ("r", _run), ("s", _segment)])


def pages_of(n):
    return (int(n) + P - 1) // P


def parts(workspace, batch, hkv, grid):
    at, out = 0, []
    for dtype, n in ((HEADER, 1), (RECORD, 2 * batch), (RUN, batch), (ROW, batch * hkv), (WARP, grid * WARPS), (CTA, grid)):
        out.append(np.frombuffer(workspace, dtype, n, at))
        at += (dtype.itemsize * n + 255) // 256 * 256
    return out


def check_plan(workspace, lens, seq_ids, prefix_ids, hq, hkv, dim, grid):
    """workspace: bytes; the rest as kv16_plan was given it (every id and length a good one)."""
    batch, g = len(prefix_ids), hq // hkv
    header, recs, runs, rows, warps, ctas = parts(workspace, batch, hkv, grid)
    h = header[0]
    assert h["magic"] == MADE and (h["batch"], h["hq"], h["hkv"], h["dim"], h["grid"]) == (batch, hq, hkv, dim, grid)
    prefix = [int(p) if p >= 0 and lens[p] > 0 else -1 for p in prefix_ids]

    # Records and runs.
    unit = col = cost = before = 0
    record, run = {}, {}
    for r in range(batch):
        n = 0
        if prefix[r] >= 0 and (r == 0 or prefix[r - 1] != prefix[r]):
            n = next((i for i in range(r, batch) if prefix[i] != prefix[r]), batch) - r
        pages = pages_of(lens[prefix[r]]) if n else 0
        small = n * g <= COLS
        record[2 * r] = dict(pages=pages if small else 0, rows=n, unit=unit, col=col, row0=r, req=prefix[r])
        if n and small:
            unit, col = unit + pages * hkv, col + n * g
        elif n:
            pair = 2 * (TILE // g)
            chunks = -(-n // pair)
            each = -(-n // chunks)
            chunks = -(-n // each)
            w = WIDE if each * g > TILE else NARROW
            run[r] = dict(pages=pages, rows=n, cost=cost, rows_before=before, chunks=chunks, each=each, w=w, len=int(lens[prefix[r]]),
                          req=prefix[r])
            cost, before = cost + (pages + OPENS[w]) * hkv * chunks * w, before + n
        own = pages_of(lens[seq_ids[r]])
        record[2 * r + 1] = dict(pages=own, rows=1, unit=unit, col=col, row0=r, req=int(seq_ids[r]))
        unit, col = unit + own * hkv, col + g
    for k, x in record.items():
        assert recs[k]["pages"] == x["pages"], k
        if x["pages"]:
            for f in x:
                assert recs[k][f] == x[f], (k, f)
    for r in range(batch):
        assert runs[r]["pages"] == (run[r]["pages"] if r in run else 0), r
        for f in ("rows", "cost", "rows_before", "chunks", "len", "req") if r in run else ():
            assert runs[r][f] == run[r][f], (r, f)

    def start(s, w):
        return w * int(s["each"]) >> 20

    for s, total in ((h["units"], unit), (h["cost"], cost)):
        assert start(s, int(s["n"])) == total and (total == 0 or s["n"] > 0)
    assert h["prefix_ctas"] == h["cost"]["n"] <= grid

    # Workers of records, as the plan starts them.
    found = {}                                   # (record, head) -> [(worker, pages, entry)]
    rec_ctas = grid - int(h["cost"]["n"])
    for w in range(rec_ctas * WARPS):
        x = warps[(int(h["cost"]["n"]) + w % rec_ctas) * WARPS + w // rec_ctas]
        if w >= h["units"]["n"]:
            assert x["count"] == 0, w
            continue
        first, stop = start(h["units"], w), start(h["units"], w + 1)
        assert (x["worker"], x["count"]) == (w, stop - first), w
        k, head, page, left = int(x["rec"]), int(x["head"]), int(x["page"]), stop - first
        assert record[k]["unit"] + head * record[k]["pages"] + page == first and page < record[k]["pages"] and head < hkv, w
        assert x["r"]["pages"] == record[k]["pages"] and x["r"]["req"] == record[k]["req"] and x["r"]["col"] == record[k]["col"], w
        while left:
            r = record[k]
            n = min(r["pages"] - page, left)
            found.setdefault((k, head), []).append((w, n, r["col"] * hkv + head * r["rows"] * g + COLS * w))
            left, page = left - n, 0
            if left:
                head += 1
                while head == hkv or record[k]["pages"] == 0:
                    k, head = k + 1, 0
    for k, r in record.items():
        for head in range(hkv if r["pages"] else 0):
            assert sum(n for _, n, _ in found[k, head]) == r["pages"], (k, head)

    # Workers of large runs.
    jobs = {}                                    # (run, job) -> [(worker, pages, entry, rows0, wide)]

    def segment(r, job, page, end, worker):
        x = run[r]
        left = end - (x["cost"] + job * (x["pages"] + OPENS[x["w"]]) * x["w"])
        stop = min(-(-left // x["w"]) - OPENS[x["w"]], x["pages"]) if left > 0 else 0
        if stop <= page:
            return None
        head, first = job // x["chunks"], job % x["chunks"] * x["each"]
        n = min(x["each"], x["rows"] - first)
        wide = n * g > TILE
        return dict(pages=stop - page, valid=x["len"] - page * P, wide=int(wide), head=head, row0=r + first, rows=n,
                    rows0=(n + 1) // 2 if wide else n, first=page,
                    entry=2 * g * (x["rows_before"] * hkv + head * x["rows"] + first) + 4 * TILE * worker)

    order = sorted(run)
    for c in range(int(h["cost"]["n"])):
        x, end = ctas[c], start(h["cost"], c + 1)
        assert x["end"] == end, c
        r = int(x["run"])
        assert r in run and all(x["r"][f] == run[r][f] for f in ("pages", "rows", "cost", "rows_before", "chunks", "len", "req")), c
        job, s = int(x["job"]), None
        if x["s"]["pages"] > 0:
            job -= 1
            s = segment(r, job, int(x["s"]["first"]), end, c)
            assert s is not None and all(x["s"][f] == s[f] for f in s), c
        while True:
            if s is not None:
                jobs.setdefault((r, job), []).append((c, s["pages"], s["entry"], s["rows0"] * g, s["wide"], s["first"]))
                job += 1
            if job >= run[r]["chunks"] * hkv:
                later = [i for i in order if i > r]
                if not later:
                    break
                r, job = later[0], 0
            s = segment(r, job, 0, end, c)
            if s is None:
                break
    for r, x in run.items():
        for job in range(x["chunks"] * hkv):
            at = 0
            for _, n, _, _, _, first in jobs[r, job]:
                assert first == at, (r, job)
                at += n
            assert at == x["pages"], (r, job)

    # Where the merge looks.
    for r in range(batch):
        first = next((i for i in order if i <= r < i + run[i]["rows"]), None)
        small = next((i for i in range(r, -1, -1) if record[2 * i]["pages"] and i <= r < i + record[2 * i]["rows"]), None)
        for kv in range(hkv):
            x = rows[r * hkv + kv]
            own = found.get((2 * r + 1, kv), [])
            assert x["own_count"] == len(own), (r, kv)
            assert [int(x["own"]) + i * COLS for i in range(len(own))] == [e for _, _, e in own], (r, kv)
            want, got = [], []
            if first is not None:
                i = run[first]
                chunk = (r - first) // i["each"]
                shift = (r - first - chunk * i["each"]) * g
                for _, _, e, second, wide, _ in jobs[first, kv * i["chunks"] + chunk]:
                    want += [e + shift] if wide else [e + shift, e + second + shift]
                assert x["stream_step"] >= 0
                for p in range(int(x["prefix_count"])):
                    two = int(x["stream_step"])
                    got.append(int(x["prefix"]) + ((p >> 1) * int(x["step"]) + (p & 1) * two if two else p * int(x["step"])))
            elif small is not None:
                want = [e + (r - small) * g for _, _, e in found[2 * small, kv]]
                assert x["stream_step"] == -1
                got = [int(x["prefix"]) + p * int(x["step"]) for p in range(int(x["prefix_count"]))]
            else:
                assert x["prefix_count"] == 0
            assert got == want, (r, kv)
