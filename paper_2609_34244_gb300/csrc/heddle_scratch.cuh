// heddle_scratch.cuh -- a context's scratch: one block that grows (plain C++).
#pragma once

#include <stddef.h>

#include <new>

namespace hd {

// Memory: static void* allocate(size_t), null where there is no room, and
// static void release(void*), which waits for the work that may use it.
template <class Memory>
class Scratch {
  public:
    Scratch() = default;
    Scratch(const Scratch&) = delete;
    Scratch& operator=(const Scratch&) = delete;

    unsigned char* get() const { return static_cast<unsigned char*>(now.p); }
    size_t size() const { return now.size; }

    // At least `need` bytes; false where there is no room, and then, with
    // `or_keep`, the block that was there stays.  A call that is `captured`
    // leaves its block's address in a graph: such a block is kept beside the
    // larger ones that follow it.  Nothing is released during a capture either,
    // which does not allow the wait.
    bool reserve(size_t need, bool captured, bool or_keep = false) {
        if (need <= now.size) {
            now.captured |= captured;
            return true;
        }
        if (!captured) release_kept(false);
        Kept* place = now.p && (captured || now.captured) ? new (std::nothrow) Kept : nullptr;
        if (now.p && (captured || now.captured) && !place) return false;
        void* p = Memory::allocate(need);
        if (!p && !place && now.p && !or_keep) {  // in the old one's room, perhaps
            Memory::release(now.p);
            now = Block{};
            p = Memory::allocate(need);
        }
        if (!p) {
            delete place;
            return false;
        }
        if (place) {
            *place = Kept{now, kept};
            kept = place;
        } else if (now.p) {
            Memory::release(now.p);
        }
        now = Block{p, need, captured};
        return true;
    }

    void release_all() {
        release_kept(true);
        if (now.p) Memory::release(now.p);
        now = Block{};
    }

  private:
    struct Block {
        void* p = nullptr;
        size_t size = 0;
        bool captured = false;
    };
    struct Kept {
        Block block;
        Kept* next = nullptr;
    };

    void release_kept(bool all) {
        for (Kept** at = &kept; *at;) {
            Kept* k = *at;
            if (!all && k->block.captured) {
                at = &k->next;
                continue;
            }
            *at = k->next;
            Memory::release(k->block.p);
            delete k;
        }
    }

    Block now;
    Kept* kept = nullptr;
};

// Room that a call can do without, once it was refused: asked for again by
// every kAgain-th call alone, since the device's refusal takes its time.
class Refusal {
  public:
    static constexpr int kAgain = 16;
    bool worth_asking(size_t need) {
        if (!least || need < least) return true;
        return ++passed % kAgain == 0;
    }
    void refused(size_t need) {
        if (least && least <= need) return;
        least = need;
        passed = 0;
    }
    void granted(size_t need) {
        if (need >= least) least = 0;
    }

  private:
    size_t least = 0;  // of the sizes refused
    unsigned passed = 0;
};

}  // namespace hd
